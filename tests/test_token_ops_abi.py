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
    # what suffices for many tokens suffices for the tables of a small model; sizes stay far from overflow
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
