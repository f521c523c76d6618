"""What the operators of a token model's sequences refuse, on the CPU: nothing is launched, the status says what kind of error it is, and
sama_op_last_error() names the call and the reason."""
import ctypes as C
import struct
import pytest
import torch

F32, BF16 = 0, 1
P = 0x10000   # stands for device memory: a refused call does not look at it
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    import os
    import paper_2310_05674_amd as pkg
    if not os.path.exists(pkg.lib_path()):
        from paper_2310_05674_amd.build import build
        build()
    return pkg.load_library()


def refused(lib, name, call, good, changes, code=1):
    """Each change alone makes the call `name` with the arguments `good` an error with a text of its own."""
    for change in changes:
        assert set(change) <= set(good), change
        rc = call(dict(good, **change))
        text = lib.sama_op_last_error().decode()
        assert rc == code and text.startswith(name + ": ") and len(text) > len(name) + 5, (change, rc, text)


def ordered(lib, name):
    return lambda args: getattr(lib, name)(*args.values())


def test_rotary_refusals(lib):
    def call(a):
        a = dict(a)
        a["sections"] = None if a["sections"] is None else (C.c_int32 * len(a["sections"]))(*a["sections"])
        return lib.sama_op_rotary(*a.values())

    good = dict(x=P, ldx=256, hsx=64, T=5, H=4, D=64, dtype=F32, positions=P, axes=2, sections=(8, 24), base=1e4, neighbours=0, inverse=0, out=P + 0x8000, ldo=256, hso=64, st=None)
    bad = [dict(dtype=2), dict(dtype=-1), dict(T=-1), dict(T=2 ** 23 + 1), dict(H=0), dict(D=1), dict(H=2 ** 15), dict(axes=0), dict(axes=5, sections=(1, 1, 1, 1, 1)),
           dict(sections=None), dict(sections=(-1, 3)), dict(sections=(0, 0)), dict(sections=(20, 13)), dict(sections=(129, 0)), dict(sections=(2 ** 31 - 1, 2 ** 31 - 1)),
           dict(base=0.0), dict(base=-1.0), dict(base=NAN), dict(base=INF), dict(neighbours=2), dict(inverse=-1), dict(x=None), dict(out=None), dict(positions=None),
           dict(positions=P + 2), dict(x=P + 2), dict(out=P + 1), dict(ldx=63), dict(hsx=63), dict(ldo=0), dict(hso=-64), dict(ldx=2 ** 62), dict(hso=2 ** 62),
           dict(out=P, ldo=320), dict(out=P, hso=128)]
    refused(lib, "sama_op_rotary", call, good, bad)
    refused(lib, "sama_op_rotary", call, dict(good, dtype=BF16), [dict(x=P + 1), dict(D=256, sections=(64, 65))])
    assert call(dict(good, T=0, x=None, out=None, positions=None)) == 0 and lib.sama_op_last_error() == b""


HEADS = ("q", "k", "v", "out", "dout", "dq", "dk", "dv")
ATTENTION = struct.Struct("@12q4P2q4i2f12q")


def attention(lib, name):
    def call(a):
        heads = [a[x] for x in HEADS]
        flat = [v for h in heads[:4] for v in h] + [a["spans"], a["at"], a["slopes"], a["lse"], a["Tq"], a["Tk"], a["Hq"], a["Hk"], a["D"], a["dtype"], a["scale"], a["cap"]]
        flat += [v for h in heads[4:] for v in h]
        return getattr(lib, name)(None if a["null"] else ATTENTION.pack(*flat), a["ws"], a["wb"], None)
    return call


def good_attention(lib, dtype, size):
    h = (P, 256, 64)
    return dict({x: h for x in HEADS}, spans=P, at=P, slopes=P, lse=P, Tq=6, Tk=6, Hq=4, Hk=2, D=64, dtype=dtype, scale=0.125, cap=0.0, null=False, ws=P, wb=size)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_refusals(lib, dtype):
    unit = 4 if dtype == F32 else 8
    for name, used in (("sama_op_attention", HEADS[:4]), ("sama_op_attention_grad", HEADS)):
        size = getattr(lib, name + "_bytes")(6, 6, 4, 2, 64, dtype)
        assert size > 0
        good, call = good_attention(lib, dtype, size), attention(lib, name)
        bad = [dict(null=True), dict(dtype=2), dict(dtype=-1), dict(Hk=0), dict(Hq=3), dict(Hq=0), dict(Hq=-2), dict(Hq=130), dict(D=0), dict(D=60), dict(D=136), dict(D=-8), dict(Tq=-1),
               dict(Tk=-1), dict(Tq=2 ** 26 + 1), dict(Tk=2 ** 27 + 1), dict(Tq=2 ** 62), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(cap=-1.0), dict(cap=NAN),
               dict(cap=INF), dict(cap=1e-4), dict(cap=5000.0), dict(spans=0), dict(spans=P + 4), dict(at=P + 2), dict(slopes=P + 1), dict(lse=P + 2), dict(at=0, Tk=7)]
        for x in used:
            bad += [{x: v} for v in ((0, 256, 64), (P + 8, 256, 64), (P, 256 + unit // 2, 64), (P, 256, 64 + unit // 2), (P, 56, 64), (P, 256, 56), (P, 0, 64), (P, -256, 64),
                                     (P, 2 ** 21 + unit, 64), (P, 256, 2 ** 41))]
        if name.endswith("grad"):
            bad += [dict(lse=0)] + [{x: (P, 256, 2 ** 29)} for x in ("q", "dout")]
        refused(lib, name, call, good, bad)
        refused(lib, name, call, good, [dict(ws=None), dict(ws=P + 128), dict(wb=0), dict(wb=size - 1)], code=3)
    assert attention(lib, "sama_op_attention")(dict(good, Tq=0, Tk=5, q=(0, 0, 0), out=(0, 0, 0), spans=0, at=0, slopes=0, lse=0)) == 0
    none = dict({x: (0, 0, 0) for x in HEADS}, spans=0, at=0, slopes=0, lse=0, Tq=0, Tk=0)
    assert attention(lib, "sama_op_attention")(dict(good, **none)) == 0 and attention(lib, "sama_op_attention_grad")(dict(good, **none)) == 0
    assert lib.sama_op_last_error() == b""


def test_attention_workspaces(lib):
    for name in ("sama_op_attention_bytes", "sama_op_attention_grad_bytes"):
        size = getattr(lib, name)
        for bad in ((-1, 1, 1, 1, 64, F32), (1, -1, 1, 1, 64, F32), (1, 1, 3, 2, 64, F32), (1, 1, 65, 1, 64, F32), (1, 1, 0, 1, 64, F32), (1, 1, 1, 0, 64, F32), (1, 1, 1, 1, 12, F32),
                    (1, 1, 1, 1, 136, F32), (1, 1, 1, 1, 64, 2), (2 ** 29, 1, 1, 1, 64, F32), (1, 2 ** 29, 1, 1, 64, BF16)):
            assert size(*bad) == 0, bad
        assert size(0, 0, 1, 1, 8, F32) > 0
        assert size(2 ** 28, 2 ** 28, 1, 1, 128, BF16) < 2 ** 38
    # parts of a long axis: 32 bits of every value and two sums of each row and part
    parts = lib.sama_op_attention_bytes(1, 100000, 4, 1, 128, BF16)
    assert parts >= 2 * 4 * (128 + 2) * 4


def test_span_refusals(lib):
    call = ordered(lib, "sama_op_attention_spans")
    good = dict(offsets=P, documents=3, prefix=None, causal=1, T=9, spans=P, st=None)
    refused(lib, "sama_op_attention_spans", call, good, [dict(documents=-1), dict(documents=2 ** 31), dict(T=-1), dict(T=2 ** 29), dict(causal=2), dict(causal=-1), dict(offsets=None), dict(spans=None),
                                                         dict(offsets=P + 2), dict(prefix=P + 1), dict(spans=P + 4)])
    assert call(dict(good, T=0, offsets=None, spans=None)) == 0 and lib.sama_op_last_error() == b""


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_distill_refusals(lib, dtype):
    call = ordered(lib, "sama_op_distill")
    good = dict(z=P, ldz=100, dtype=dtype, T=5, V=100, ids=P, teacher=P, K=8, tau=2.0, loss=P, saved=P, st=None)
    bad = [dict(dtype=2), dict(dtype=-1), dict(T=-1), dict(T=2 ** 22 + 1), dict(V=0), dict(V=-3), dict(K=0), dict(K=257), dict(tau=0.0), dict(tau=-1.0), dict(tau=NAN), dict(tau=INF), dict(tau=1e-5), dict(tau=2e4),
           dict(z=None), dict(ids=None), dict(teacher=None), dict(ids=P + 2), dict(teacher=P + 1), dict(ldz=99), dict(ldz=2 ** 60), dict(z=P + 1), dict(loss=None), dict(saved=None), dict(loss=P + 2),
           dict(saved=P + 3)]
    refused(lib, "sama_op_distill", call, good, bad)
    assert call(dict(good, T=0, z=None, ids=None, teacher=None, loss=None, saved=None)) == 0
    call = ordered(lib, "sama_op_distill_grad")
    good = dict(z=P, ldz=100, dtype=dtype, T=5, V=100, ids=P, teacher=P, K=8, tau=2.0, dloss=P, saved=P, dz=P + 0x10000, lddz=100, st=None)
    bad = [dict(dtype=3), dict(T=-1), dict(V=0), dict(K=0), dict(K=300), dict(tau=0.0), dict(z=None), dict(ids=None), dict(teacher=None), dict(ldz=99), dict(dloss=None), dict(dloss=P + 2), dict(saved=None),
           dict(saved=P + 1), dict(dz=None), dict(dz=P + 1), dict(lddz=99), dict(lddz=2 ** 60), dict(dz=P, lddz=104)]
    refused(lib, "sama_op_distill_grad", call, good, bad)
    assert call(dict(good, T=0, z=None, ids=None, teacher=None, dloss=None, saved=None, dz=None)) == 0
    assert lib.sama_op_last_error() == b""


def test_binding_wants_tensors_of_the_gpu(lib):
    """Tensors that are not on the current GPU never reach the library."""
    from paper_2310_05674_amd import binding as B
    x = torch.zeros(4, 2, 64)
    n = torch.zeros(4, dtype=torch.int32)
    spans = torch.zeros(4, 2, dtype=torch.int32)
    z, teacher = torch.zeros(4, 10), torch.zeros(4, 3)
    ids, loss, saved = torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4), torch.zeros(4, 2)
    ws = torch.zeros(4096, dtype=torch.uint8)
    for call in (lambda: B.op_rotary(x, n, x), lambda: B.op_attention_spans(n, spans), lambda: B.op_attention(x, x, x, x, spans, ws),
                 lambda: B.op_attention_grad(x, x, x, x, x, z, spans, x, x, x, ws), lambda: B.op_distill(z, ids, teacher, loss, saved),
                 lambda: B.op_distill_grad(z, ids, teacher, loss, saved, z)):
        with pytest.raises(ValueError, match="current GPU"):
            call()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_single_token_has_no_stride_between_tokens(lib, dtype):
    """One token of [heads][tokens][width] memory of a long text: what lies between its heads is no stride between tokens, which has a limit."""
    from paper_2310_05674_amd import binding as B
    H, D = 2, 128
    whole = torch.empty(H, 16640, D, dtype=dtype).transpose(0, 1)
    code, between = {torch.float32: F32, torch.bfloat16: BF16}[dtype], 16640 * D
    for view in (whole[100:101], whole[:0]):
        p, ld, hs = B._heads(view, view.shape, dtype, -1, "q")
        assert (ld, hs) == (D, between)
    assert B._heads(whole[100:102], (2, H, D), dtype, -1, "q")[1:] == (D, between) and B._heads(whole[5:6, 1:], (1, 1, D), dtype, -1, "q")[1:] == (D, D)
    # every stride of such a token is one that the call takes: what it refuses is the workspace alone
    one = (P, *B._heads(whole[100:101], (1, H, D), dtype, -1, "q")[1:])
    for name in ("sama_op_attention", "sama_op_attention_grad"):
        good = dict(good_attention(lib, code, 0), D=D, Hq=H, Hk=H, Tq=1, Tk=1, **{x: one for x in HEADS})
        refused(lib, name, attention(lib, name), good, [dict(ws=None)], code=3)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_refuses_more_key_heads_than_a_launch_has_workgroups(lib, dtype):
    """One token of 2^20 + 1 key heads and more is within Tq Hq <= 2^28, but their workgroups may be more work items than a launch holds."""
    for name in ("sama_op_attention", "sama_op_attention_grad"):
        size = getattr(lib, name + "_bytes")
        assert size(1, 1, 2 ** 20, 2 ** 20, 64, dtype) > 0
        good = dict(good_attention(lib, dtype, 2 ** 40), Tq=1, Tk=1)
        bad = [dict(Hq=h, Hk=h) for h in (2 ** 20 + 1, 2 ** 24, 2 ** 28)]
        refused(lib, name, attention(lib, name), good, bad)
        assert all(size(1, 1, b["Hq"], b["Hk"], 64, dtype) == 0 for b in bad)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_distill_refuses_rows_whose_last_pieces_pass_32_bits(lib, dtype):
    """A thread's place in a row is a 32-bit number, and the last one's is up to 4 x 1024 pieces behind the row's end."""
    good = dict(z=P, ldz=2 ** 31, dtype=dtype, T=1, V=100, ids=P, teacher=P, K=8, tau=2.0, loss=P, saved=P, st=None)
    bad = [dict(V=v) for v in (2 ** 30 + 1, 2 ** 31 - 1024, 2 ** 31 - 1)]
    refused(lib, "sama_op_distill", ordered(lib, "sama_op_distill"), good, bad)
    good = dict(z=P, ldz=2 ** 31, dtype=dtype, T=1, V=100, ids=P, teacher=P, K=8, tau=2.0, dloss=P, saved=P, dz=P + 0x10000, lddz=2 ** 31, st=None)
    refused(lib, "sama_op_distill_grad", ordered(lib, "sama_op_distill_grad"), good, bad)


def test_rotary_refuses_bases_whose_angles_have_no_fraction(lib):
    """Rates grow with the pair where the base is below 1: at 1e-6 the last position's 2^48 turns have 4 bits behind the point, far below that an angle is infinite and its sine no number."""
    def call(a):
        a = dict(a)
        a["sections"] = (C.c_int32 * len(a["sections"]))(*a["sections"])
        return lib.sama_op_rotary(*a.values())

    assert 2.0 ** 31 * 1e-6 ** (-126 / 128) / 6.28 < 2.0 ** 49 and 5e-324 == 2.0 ** -1074 and 1074 * 126 / 128 > 1024
    good = dict(x=P, ldx=512, hsx=128, T=5, H=4, D=128, dtype=F32, positions=P, axes=1, sections=(64,), base=1e4, neighbours=0, inverse=0, out=P + 0x8000, ldo=512, hso=128, st=None)
    refused(lib, "sama_op_rotary", call, good, [dict(base=b) for b in (9.9e-7, 1e-100, 1e-300, 5e-324)])
    for base in (1e-6, 0.5, 1.0, 1.7e308):
        assert call(dict(good, T=0, base=base)) == 0


@pytest.mark.parametrize("dtype,D,places", [(BF16, 128, 256), (F32, 64, 256), (F32, 128, 256), (BF16, 64, 512), (BF16, 32, 512), (BF16, 72, 256)])
def test_split_keys_fill_the_chip_once_or_twice(lib, dtype, D, places):
    """The parts of split keys, from the workspace's size: as many workgroups as fit the chip at once, of 128 KB each or (bf16, widths up to 64) 64 KB, where two rounds of them would not do
    with much shorter parts."""
    def parts(heads, Tk):
        size = lib.sama_op_attention_bytes(1, Tk, heads, heads, D, dtype)
        each = heads * (D + 1) * 4
        assert size == 256 or size % each == 0
        return 1 if size == 256 else size // each

    for heads in range(1, 257):
        one, two = places // heads, 2 * places // heads
        for Tk in (1, 511, 1023, 1024, 5000, 100000):
            n, most = parts(heads, Tk), max(1, min(64, Tk // 512))
            twice = one <= 2 and two > 2 * one and Tk >= 1024 * two
            assert n == max(1, min(most, two if twice else one)), (heads, Tk, n)
    assert parts(257, 100000) == 1
