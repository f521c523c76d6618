"""What the operators of a token model's step refuse, on the CPU: nothing is launched, the status says what kind of error it is, and
sama_op_last_error() names the call and the reason."""
import ctypes as C
import pytest

F32, BF16 = 0, 1
P = 0x10000   # stands for device memory: a refused call does not look at it


@pytest.fixture(scope="module")
def lib():
    import os
    import paper_2310_05674_amd as pkg
    if not os.path.exists(pkg.lib_path()):
        from paper_2310_05674_amd.build import build
        build()
    return pkg.load_library()


def refused(lib, name, good, changes, code=1):
    """Each change alone makes the call `name` with the arguments `good` an error with a text of its own."""
    keys = list(good)
    for change in changes:
        args = dict(good, **change)
        rc = getattr(lib, name)(*[args[k] for k in keys])
        text = lib.sama_op_last_error().decode()
        assert rc == code and text.startswith(name + ": ") and len(text) > len(name) + 5, (change, rc, text)


def test_embedding_refusals(lib):
    good = dict(table=P, tt=F32, ldt=64, ids=P, n=3, V=10, d=64, scale=1.0, pad=-1, out=P, ot=BF16, ldo=64, st=None)
    refused(lib, "sama_op_embedding", good,
            [dict(tt=2), dict(ot=-1), dict(n=-1), dict(n=2 ** 30 + 1), dict(V=0), dict(d=0), dict(ids=None), dict(ids=P + 2), dict(scale=float("nan")),
             dict(scale=float("inf")), dict(pad=-2), dict(table=None), dict(out=None), dict(ldt=63), dict(ldo=0), dict(table=P + 2), dict(out=P + 1),
             dict(ldo=2 ** 50), dict(ldt=2 ** 41)])
    assert lib.sama_op_embedding(*dict(good, n=0, table=None, out=None, ids=None).values()) == 0
    assert lib.sama_op_last_error() == b""


def test_embedding_gradient_refusals(lib):
    size = lib.sama_op_embedding_grad_bytes(3, 10, 64)
    assert size > 0
    good = dict(dy=P, dt=F32, ldy=64, ids=P, n=3, V=10, d=64, scale=1.0, pad=-1, acc=0, grad=P, gt=F32, ldg=64, ws=P, wb=size, st=None)
    refused(lib, "sama_op_embedding_grad", good,
            [dict(dt=7), dict(gt=2), dict(n=-1), dict(n=2 ** 31), dict(V=0), dict(d=-5), dict(ids=None), dict(scale=float("nan")), dict(pad=-7), dict(acc=2),
             dict(dy=None), dict(grad=None), dict(ldy=10), dict(ldg=63), dict(grad=P + 2), dict(dy=P + 3), dict(ldy=2 ** 45)])
    refused(lib, "sama_op_embedding_grad", good, [dict(ws=None), dict(ws=P + 128), dict(wb=size - 1), dict(wb=0)], code=3)
    assert lib.sama_op_embedding_grad(*dict(good, n=0, acc=1, dy=None, ids=None).values()) == 0
    for bad in ((-1, 10, 64), (2 ** 30 + 1, 10, 64), (3, 0, 64), (3, 10, 0)):
        assert lib.sama_op_embedding_grad_bytes(*bad) == 0
    sizes = [lib.sama_op_embedding_grad_bytes(n, 5000, 768) for n in list(range(0, 9000, 37)) + [20000, 65536, 10 ** 6]]
    assert sizes == sorted(sizes)                     # what suffices for many tokens suffices for fewer
    assert lib.sama_op_embedding_grad_bytes(2 ** 30, 2 ** 31 - 1, 1024) > 2 ** 33


def test_clipping_refusals(lib):
    def call(count=2, grads=(P, P), counts=(5, 6), dtypes=(F32, BF16), max_norm=1.0, out=None, norm=P, status=None, ws=P, wb=lib.sama_op_grad_clip_bytes(),
             lists=True):
        k = len(grads)
        a = ((C.c_void_p * k)(*grads), (C.c_int64 * k)(*counts), (C.c_int32 * k)(*dtypes)) if lists else (None, None, None)
        return lib.sama_op_grad_clip(count, *a, max_norm, out, norm, status, ws, wb, None), lib.sama_op_last_error().decode()

    for bad in (dict(count=-1), dict(lists=False), dict(dtypes=(F32, 2)), dict(counts=(5, -1)), dict(counts=(5, 2 ** 41)), dict(counts=(2 ** 40, 2)), dict(grads=(P, None)), dict(grads=(P + 2, P)),
                dict(grads=(P, P + 1)), dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(norm=None), dict(norm=P + 2),
                dict(out=P + 1), dict(status=P + 4)):
        rc, text = call(**bad)
        assert rc == 1 and text.startswith("sama_op_grad_clip: "), (bad, rc, text)
    for bad in (dict(ws=None), dict(ws=P + 64), dict(wb=lib.sama_op_grad_clip_bytes() - 1)):
        rc, text = call(**bad)
        assert rc == 3 and text.startswith("sama_op_grad_clip: "), (bad, rc, text)


def test_feed_forward_refusals(lib):
    T, d, F = 5, 64, 72
    for dtype in (BF16, F32):
        size, saved = lib.sama_op_glu_ffn_bytes(T, d, F, dtype), lib.sama_op_glu_ffn_saved_bytes(T, F, dtype)
        assert size > 0 and saved > 0
        good = dict(x=P, ldx=64, wi=P, wo=P, T=T, d=d, F=F, act=0, dtype=dtype, y=P, ldy=64, hidden=P, saved=None, ws=P, wb=size, st=None)
        bad = [dict(T=-1), dict(T=2 ** 22 + 1), dict(d=0), dict(F=-8), dict(d=2 ** 15, F=2 ** 14), dict(act=2), dict(act=-1), dict(dtype=2), dict(x=None), dict(y=None),
               dict(wi=None), dict(wo=None), dict(hidden=None), dict(ldx=63), dict(ldy=56), dict(ldx=2 ** 22), dict(x=P + 1), dict(saved=P + 4)]
        if dtype == BF16:
            bad += [dict(d=60), dict(F=70), dict(ldx=68), dict(ldy=66), dict(x=P + 8), dict(wi=P + 8), dict(wo=P + 4), dict(hidden=P + 2), dict(y=P + 8)]
        refused(lib, "sama_op_glu_ffn", good, bad)
        refused(lib, "sama_op_glu_ffn", good, [dict(ws=None), dict(ws=P + 16), dict(wb=size - 1)], code=3)
        assert lib.sama_op_glu_ffn(*dict(good, T=0, x=None, y=None, hidden=None).values()) == 0
        size = lib.sama_op_glu_ffn_grad_bytes(T, d, F, dtype)
        good = dict(dy=P, lddy=64, x=P, ldx=64, wi=P, wo=P, hidden=P, saved=P, T=T, d=d, F=F, act=1, dtype=dtype, dx=P, lddx=64, dwi=P, dwo=P, dwt=dtype, ws=P, wb=size,
                    st=None)
        bad = [dict(T=-1), dict(d=-64), dict(act=9), dict(dtype=-1), dict(dy=None), dict(x=None), dict(dx=None), dict(wi=None), dict(wo=None), dict(hidden=None), dict(saved=None),
               dict(saved=P + 8), dict(dwi=None), dict(dwo=None), dict(lddy=10), dict(lddx=63), dict(dwt=3), dict(dwt=-1)]
        bad += [dict(dwt=BF16)] if dtype == F32 else [dict(dx=P + 8), dict(lddy=68), dict(dwi=P + 8), dict(F=4)]
        refused(lib, "sama_op_glu_ffn_grad", good, bad)
        refused(lib, "sama_op_glu_ffn_grad", good, [dict(ws=None), dict(ws=P + 16), dict(wb=size - 1)], code=3)
    for f in (lib.sama_op_glu_ffn_bytes, lib.sama_op_glu_ffn_grad_bytes):
        assert f(-1, 64, 72, BF16) == f(5, 60, 72, BF16) == f(5, 64, 72, 2) == f(5, 2 ** 15, 2 ** 14, F32) == 0
        for dtype in (BF16, F32):
            sizes = [f(T, 520, 1368, dtype) for T in list(range(0, 3000, 23)) + [8192, 65536, 2 ** 22]]
            assert sizes == sorted(sizes)             # what suffices for many tokens suffices for fewer
            assert f(2 ** 22, 4096, 16384, dtype) > 0


def test_sizes_beyond_a_launch(lib):
    """Sizes whose offsets or launches would not fit 32 bits are refused, whatever the workspace."""
    grad = dict(dy=P, dt=F32, ldy=2 ** 16, ids=P, n=2 ** 30, V=10, d=2 ** 16, scale=1.0, pad=-1, acc=0, grad=P, gt=F32, ldg=2 ** 16, ws=P, wb=2 ** 62, st=None)
    refused(lib, "sama_op_embedding_grad", grad, [dict(), dict(d=1), dict(dt=BF16), dict(n=3, d=64, V=2 ** 30 + 1)])
    for dtype in (BF16, F32):
        for d, F in ((8, 2 ** 20 + 8), (2 ** 20 + 8, 8), (2 ** 15, 2 ** 14) if dtype == BF16 else (2 ** 14, 2 ** 14)):
            up = dict(x=P, ldx=2 ** 21, wi=P, wo=P, T=5, d=d, F=F, act=0, dtype=dtype, y=P, ldy=2 ** 21, hidden=P, saved=None, ws=P, wb=2 ** 62, st=None)
            refused(lib, "sama_op_glu_ffn", up, [dict()])
            down = dict(dy=P, lddy=2 ** 21, x=P, ldx=2 ** 21, wi=P, wo=P, hidden=P, saved=P, T=5, d=d, F=F, act=0, dtype=dtype, dx=P, lddx=2 ** 21, dwi=P, dwo=P,
                        dwt=dtype, ws=P, wb=2 ** 62, st=None)
            refused(lib, "sama_op_glu_ffn_grad", down, [dict()])
            assert lib.sama_op_glu_ffn_bytes(5, d, F, dtype) == lib.sama_op_glu_ffn_grad_bytes(5, d, F, dtype) == 0
        assert lib.sama_op_glu_ffn_bytes(5, 8, 2 ** 20, dtype) > 0 and lib.sama_op_glu_ffn_grad_bytes(5, 2 ** 20, 8, dtype) > 0


def test_tile_switch_refusals(lib):
    """The development switch takes the tiles that there are, alone or with a number of parts; anything else is refused and changes nothing."""
    try:
        for tile in (32, 64, 128, 192, 256, 3064, 16256, 4000, 0):
            assert lib.sama_dev_glu_tile(tile) == 0, tile
        for tile in (1, 16, 31, 33, 96, 127, 129, 255, 257, 512, 999, 1001, 2100, 3065, -1, -32, -64, -1000, -3064, 2 ** 31 - 1, -2 ** 31):
            assert lib.sama_dev_glu_tile(tile) == 1, tile
    finally:
        lib.sama_dev_glu_tile(0)
