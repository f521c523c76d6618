"""The gated feed-forward block against its formulas in 64 bits.

Tolerances.  u = 2^-24 is the unit roundoff of fp32 and 2^-8 that of bf16.  A sum of K products in fp32 is within (K + 2) u of the sum of their
sizes; what that does to a later value is followed through the formulas to first order, by the same products of absolute values
(bars() below).  In bf16 h, dg, du and every output are rounded once more, each value by at most 2^-8 of itself, and g and u reach the
backward pass with 2^-15.  The gate's exp, erf and reciprocal are good to 1e-6 of its size.  On top of the bar for each value, rounding errors
that have no reason to agree add up like their root mean square, 1.66e-3 for a value spread over a binade: two roundings 2.35e-3 of the norm, and
3e-3 is what the norm of an error may be where there are a thousand values and more."""
import math
import numpy as np
import pytest
import torch
from datagen import CounterRNG

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32, U16, U24 = 2.0 ** -24, 2.0 ** -8, 2.0 ** -15
T_ = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True)
def heuristic_afterwards():
    yield
    import paper_2310_05674_amd as pkg
    pkg.load_library().sama_dev_glu_tile(0)


def values(seed, rows, cols, std, dtype):
    v = CounterRNG(seed).normal(1, rows * cols).reshape(rows, cols).astype(np.float32) * std
    return torch.as_tensor(v, device=DEV).to(dtype)


def inputs(T, d, F, dtype, seed=0):
    t = T_[dtype]
    return dict(x=values(seed + 1, T, d, 1.0, t), w_in=values(seed + 2, 2 * F, d, d ** -0.5, t), w_out=values(seed + 3, d, F, F ** -0.5, t),
                dy=values(seed + 4, T, d, 1.0, t))


def gate64(act, g):
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s + g * s * (1 - s)
    P = 0.5 * torch.erfc(-g / math.sqrt(2))
    return g * P, P + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def exact(i, act):
    """Values in 64 bits and a bar for each (bars of `bf16` and of `fp32` from the same expressions)."""
    bf = i["x"].dtype == torch.bfloat16
    r16, r24 = (U16 * 1.01, U24) if bf else (0.0, 0.0)
    x, wi, wo, dy = (i[k].double() for k in ("x", "w_in", "w_out", "dy"))
    F, d, T = wo.shape[1], x.shape[1], x.shape[0]
    out = U16 * 1.01 if bf else U32
    mm = torch.mm
    pre, dpre_ = mm(x, wi.t()), (d + 2) * U32 * mm(x.abs(), wi.abs().t())
    g, u, eg, eu = pre[:, :F], pre[:, F:], dpre_[:, :F], dpre_[:, F:]
    a, da = gate64(act, g)
    fn = 1e-6 if bf else 8 * U32           # exp, erf, reciprocal: a few roundings; bf16: fast ones
    ea, eda = da.abs() * eg + fn * (a.abs() + g.abs() * 0.1), 1.2 * (eg + r24 * g.abs()) + fn * 2
    h = a * u
    eh = ea * u.abs() + a.abs() * eu + (r16 + 2 * U32) * h.abs()
    y = mm(h, wo.t())
    ey = mm(eh, wo.abs().t()) + (F + 2) * U32 * mm(h.abs(), wo.abs().t())
    dh, edh = mm(dy, wo), (d + 2) * U32 * mm(dy.abs(), wo.abs())
    dg, du = dh * da * u, dh * a
    ea2 = ea + da.abs() * r24 * g.abs()
    edg = edh * (da * u).abs() + (dh * u).abs() * eda + (dh * da).abs() * (eu + r24 * u.abs()) + (r16 + 4 * U32) * dg.abs()
    edu = edh * a.abs() + dh.abs() * ea2 + (r16 + 2 * U32) * du.abs()
    dp, edp = torch.cat([dg, du], 1), torch.cat([edg, edu], 1)
    dx = mm(dp, wi)
    edx = mm(edp, wi.abs()) + (2 * F + 2) * U32 * mm(dp.abs(), wi.abs())
    dwi, edwi = mm(dp.t(), x), mm(edp.t(), x.abs()) + (T + 2) * U32 * mm(dp.abs().t(), x.abs())
    dwo, edwo = mm(dy.t(), h), mm(dy.abs().t(), eh) + (T + 2) * U32 * mm(dy.abs().t(), h.abs())
    return {k: (v, e + (out if k in ("y", "dx") or bf else U32) * v.abs() + 1e-37) for k, v, e in
            (("y", y, ey), ("hidden", h, eh), ("dx", dx, edx), ("dw_in", dwi, edwi), ("dw_out", dwo, edwo))}


def strided(T, d, ld, dtype, fill=7.0):
    whole = torch.full((max(T, 1) * ld + 64,), fill, device=DEV, dtype=dtype)
    return whole[:T * ld].view(T, ld)[:, :d], whole


def run(i, act, *, train=True, ld=None, dw="same"):
    from paper_2310_05674_amd import binding as B
    x, wi, wo, dy = i["x"], i["w_in"], i["w_out"], i["dy"]
    (T, d), F, t = x.shape, wo.shape[1], x.dtype
    ld = d if ld is None else ld
    scratch = lambda n: torch.full((n,), 0xff, dtype=torch.uint8, device=DEV)   # NaN, in every type
    nan = float("nan")
    (y, yw), (dx, dxw) = strided(T, d, ld, t), strided(T, d, ld, t)
    hidden = torch.full((T, F), nan, device=DEV, dtype=t)
    saved = scratch(B.glu_ffn_saved_bytes(T, F, t)) if train else None
    B.op_glu_ffn(x, wi, wo, y, hidden, scratch(B.glu_ffn_bytes(T, d, F, t)), act=act, saved=saved)
    out = dict(y=y, hidden=hidden)
    if train:
        wt = torch.float32 if dw == "fp32" else t
        dwi, dwo = torch.full((2 * F, d), nan, device=DEV, dtype=wt), torch.full((d, F), nan, device=DEV, dtype=wt)
        B.op_glu_ffn_grad(dy, x, wi, wo, hidden, saved, dx, dwi, dwo, scratch(B.glu_ffn_grad_bytes(T, d, F, t)), act=act)
        out.update(dx=dx, dw_in=dwi, dw_out=dwo)
    for w in (yw, dxw) if train else (yw,):       # nothing beside the rows
        assert bool((w[T * ld:] == 7.0).all())
        if T and ld > d:
            assert bool((w[:T * ld].view(T, ld)[:, d:] == 7.0).all())
    return out


def check(got, want, bf):
    for k, v in got.items():
        w, bar = want[k]
        off = (v.double() - w).abs()
        assert bool((off <= bar).all()), (k, float((off / bar).max()), int((~(off <= bar)).sum()))
        if bf and w.numel() >= 1000:
            assert float(off.norm() / w.norm()) <= 3e-3, k


SHAPES = [(1, 8, 8), (2, 64, 64), (7, 16, 24), (8, 200, 520), (9, 72, 40), (16, 128, 136), (17, 264, 1032), (33, 520, 200), (64, 64, 128), (65, 136, 72), (130, 192, 328),
          (257, 256, 512), (300, 72, 1368), (513, 328, 264)]


@pytest.mark.parametrize("tile", [0, 32, 64, 128, 192, 256, 3064])
@pytest.mark.parametrize("T,d,F", SHAPES)
def test_bf16(T, d, F, tile):
    import paper_2310_05674_amd as pkg
    pkg.load_library().sama_dev_glu_tile(tile)
    act = "silu" if (T + d) % 3 else "gelu"
    i = inputs(T, d, F, "bf16", T)
    got = run(i, act, ld=d + 8 * (T % 3))
    check(got, exact(i, act), True)
    again = run(i, act, ld=d + 8 * (T % 3))
    assert all(torch.equal(got[k], again[k]) for k in got)                 # a fixed order
    alone = run(i, act, train=False)
    assert torch.equal(alone["y"], got["y"])


@pytest.mark.parametrize("tile", [0, 32, 64, 128, 192, 256, 2032, 5064, 3128, 4192, 2256, 16256])
@pytest.mark.parametrize("T,d,F", [(8, 64, 8192), (100, 128, 4104), (2100, 64, 72), (1000, 136, 3000), (4100, 256, 256), (700, 1024, 512)])
def test_bf16_split_contractions(T, d, F, tile):
    """Few tiles and long contractions: sums over several workgroups, in every product that may be cut."""
    import paper_2310_05674_amd as pkg
    pkg.load_library().sama_dev_glu_tile(tile)
    i = inputs(T, d, F, "bf16", T + 1)
    got = run(i, "silu", dw="fp32")
    check(got, exact(i, "silu"), True)
    again = run(i, "silu", dw="fp32")
    assert all(torch.equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T,d,F", [(1, 1, 1), (3, 5, 7), (16, 64, 100), (65, 33, 130), (128, 256, 688), (301, 100, 173)])
def test_fp32(T, d, F, act):
    i = inputs(T, d, F, "fp32", T)
    got = run(i, act, ld=d + T % 2)
    check(got, exact(i, act), False)
    again = run(i, act)
    assert all(torch.equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("tile", [32, 64, 128, 256, 4032, 2064, 7128])
@pytest.mark.parametrize("T,d,F", [(1, 4, 4), (5, 12, 20), (33, 100, 36), (64, 64, 128), (130, 36, 1368), (257, 260, 132), (2100, 64, 68), (700, 256, 2000)])
def test_fp32_tiles(T, d, F, tile):
    import paper_2310_05674_amd as pkg
    pkg.load_library().sama_dev_glu_tile(tile)
    act = "silu" if T % 2 else "gelu"
    i = inputs(T, d, F, "fp32", T)
    got = run(i, act, ld=d + 4 * (T % 3))
    check(got, exact(i, act), False)
    again = run(i, act)
    assert all(torch.equal(got[k], again[k]) for k in got)


def test_fp32_forward_and_backward_of_other_alignment():
    """A forward call whose x begins at any float, and a backward call on an aligned copy of it."""
    from paper_2310_05674_amd import binding as B
    T, d, F = 90, 64, 72
    i = inputs(T, d, F, "fp32", 2)
    whole = torch.zeros(T * d + 1, device=DEV)
    odd = whole[1:].view(T, d)
    odd.copy_(i["x"])
    scratch = lambda n: torch.empty(n, dtype=torch.uint8, device=DEV)
    e = lambda *s: torch.empty(*s, device=DEV)
    t = torch.float32
    for first, second in ((odd, i["x"]), (i["x"], odd)):
        y, hidden, saved, dx, dwi, dwo = e(T, d), e(T, F), scratch(B.glu_ffn_saved_bytes(T, F, t)), e(T, d), e(2 * F, d), e(d, F)
        B.op_glu_ffn(first, i["w_in"], i["w_out"], y, hidden, scratch(B.glu_ffn_bytes(T, d, F, t)), saved=saved)
        B.op_glu_ffn_grad(i["dy"], second, i["w_in"], i["w_out"], hidden, saved, dx, dwi, dwo, scratch(B.glu_ffn_grad_bytes(T, d, F, t)))
        check(dict(y=y, hidden=hidden, dx=dx, dw_in=dwi, dw_out=dwo), exact(i, "silu"), False)


@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 6, 7, 8, 9, 12, 16, 17, 24, 31, 32, 48, 63, 64])
@pytest.mark.parametrize("d,F", [(768, 2048), (1024, 4096), (520, 1368)])
def test_few_tokens(T, d, F):
    """The sizes of serving, one token at a time and a few."""
    act = "gelu" if T % 2 else "silu"
    i = inputs(T, d, F, "bf16", T)
    check(run(i, act, train=False), exact(i, act), True)


def test_rows_do_not_touch_one_another():
    """A token of NaN and infinities, and weights' columns beside the matrix: the other tokens keep their bits."""
    for T, d, F in ((5, 136, 200), (70, 200, 136), (300, 136, 328)):
        i = inputs(T, d, F, "bf16", 9)
        clean = run(i, "silu", train=False)
        bad = T // 2
        i["x"][bad] = float("nan"); i["x"][bad, 0] = float("inf")
        got = run(i, "silu")
        keep = torch.arange(T, device=DEV) != bad
        assert torch.equal(got["y"][keep], clean["y"][keep]) and torch.equal(got["hidden"][keep], clean["hidden"][keep])
        assert bool(torch.isnan(got["y"][bad].float()).all()) and bool(torch.isfinite(got["dx"][keep].float()).all())


def test_large_gates():
    """Where the gate is 0 or its argument, and where exp leaves the range of fp32."""
    T, d, F = 64, 64, 128
    for act in ("silu", "gelu"):
        i = inputs(T, d, F, "bf16", 3)
        i["w_in"][:F] *= 100.0
        got, want = run(i, act), exact(i, act)
        for k in got:
            assert bool(torch.isfinite(got[k].float()).all())
            assert float((got[k].double() - want[k][0]).norm() / want[k][0].norm()) <= 3e-3, (act, k)


def test_zero_tokens():
    for dtype in ("bf16", "fp32"):
        i = inputs(0, 64, 72, dtype)
        got = run(i, "silu", dw="fp32")
        assert not got["dw_in"].any() and not got["dw_out"].any()
        got = run(i, "silu")
        assert not got["dw_in"].any() and not got["dw_out"].any()


def test_inputs_with_strides():
    T, d, F = 77, 128, 200
    i = inputs(T, d, F, "bf16", 1)
    want = run(i, "gelu")
    for name, ld in (("x", 136), ("dy", 192)):
        wide, _ = strided(T, d, ld, torch.bfloat16, fill=float("nan"))     # what lies between the rows is not read into anything
        wide.copy_(i[name])
        i[name] = wide
    got = run(i, "gelu")
    assert all(torch.equal(got[k], want[k]) for k in want)


def test_fp32_gradient_against_differences():
    """(L(p + e E) - L(p - e E)) / 2 e of the operator's own forward pass against <gradient, E>, L = <dy, y>.  How far such a quotient is from the derivative
    is taken from the same quotient in 64 bits; the rest is fp32 rounding of the two passes, a relative (d + F) u of sums of sizes, over e."""
    T, d, F, e = 40, 48, 72, 2.0 ** -6
    for act in ("silu", "gelu"):
        i = inputs(T, d, F, "fp32", 5)
        grads = run(i, act)
        for name, grad in (("x", "dx"), ("w_in", "dw_in"), ("w_out", "dw_out")):
            E = values(50, *i[name].shape, 1.0 if name == "x" else 0.1, torch.float32)
            both = {}
            size = 0.0
            for s in (1, -1):
                j = dict(i, **{name: i[name] + s * e * E})
                w, bar = exact(j, act)["y"]
                both[s] = (float((run(j, act, train=False)["y"].double() * i["dy"].double()).sum()), float((w * i["dy"].double()).sum()))
                size += float((bar * i["dy"].double().abs()).sum())
            got, wide = ((both[1][k] - both[-1][k]) / (2 * e) for k in (0, 1))
            assert abs(got - wide) <= size / (2 * e)
            slope = float((exact(i, act)[grad][0] * E.double()).sum())
            mine = float((grads[grad].double() * E.double()).sum())
            bar = float((exact(i, act)[grad][1] * E.double().abs()).sum())
            assert abs(mine - slope) <= bar
            assert abs(got - mine) <= abs(wide - slope) + size / (2 * e) + bar


def test_in_a_graph_and_on_another_stream():
    from paper_2310_05674_amd import binding as B
    T, d, F = 300, 192, 328
    t = torch.bfloat16
    i = inputs(T, d, F, "bf16", 1)
    e = lambda *s: torch.zeros(*s, device=DEV, dtype=t)
    scratch = lambda n: torch.empty(n, dtype=torch.uint8, device=DEV)
    hidden, y, dx, dwi, dwo = e(T, F), e(T, d), e(T, d), e(2 * F, d), e(d, F)
    saved, ws, wg = scratch(B.glu_ffn_saved_bytes(T, F, t)), scratch(B.glu_ffn_bytes(T, d, F, t)), scratch(B.glu_ffn_grad_bytes(T, d, F, t))
    outs = (y, dx, dwi, dwo)

    def step():
        B.op_glu_ffn(i["x"], i["w_in"], i["w_out"], y, hidden, ws, saved=saved)
        B.op_glu_ffn_grad(i["dy"], i["x"], i["w_in"], i["w_out"], hidden, saved, dx, dwi, dwo, wg)

    step()
    want = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for o in outs:
            o.fill_(5.0)
        step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        i["x"].copy_(values(60 + k, T, d, 1.0, t)); i["dy"].copy_(values(70 + k, T, d, 1.0, t))
        step()
        want = [o.clone() for o in outs]
        for o in outs:
            o.fill_(5.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), k


def test_what_the_binding_refuses():
    """On the host, other types or shapes, an unknown gate: an error that launches nothing."""
    from paper_2310_05674_amd import binding as B
    T, d, F = 5, 64, 72
    new = lambda *s, dtype=torch.bfloat16, device=DEV: torch.zeros(*s, dtype=dtype, device=device)
    good = dict(x=new(T, d), w_in=new(2 * F, d), w_out=new(d, F), y=new(T, d), hidden=new(T, F), ws=new(B.glu_ffn_bytes(T, d, F, torch.bfloat16), dtype=torch.uint8), act="silu",
                saved=new(B.glu_ffn_saved_bytes(T, F, torch.bfloat16), dtype=torch.uint8))

    def forward(**change):
        a = dict(good, **change)
        B.op_glu_ffn(a["x"], a["w_in"], a["w_out"], a["y"], a["hidden"], a["ws"], act=a["act"], saved=a["saved"])

    forward()
    for k in ("x", "w_in", "w_out", "y", "hidden", "ws", "saved"):
        with pytest.raises(ValueError):
            forward(**{k: good[k].cpu()})
    for bad in (dict(w_in=new(F, d)), dict(y=new(T + 1, d)), dict(y=new(T, d, dtype=torch.float32)), dict(hidden=new(T, F + 8)), dict(saved=good["saved"][:-1]), dict(x=new(T, 2 * d)[:, ::2])):
        with pytest.raises(ValueError):
            forward(**bad)
    for bad in (dict(act="relu"), dict(ws=good["ws"][:-1])):
        with pytest.raises(B.SamaError):
            forward(**bad)
    back = dict(dy=new(T, d), dx=new(T, d), dwi=new(2 * F, d), dwo=new(d, F), ws=new(B.glu_ffn_grad_bytes(T, d, F, torch.bfloat16), dtype=torch.uint8))

    def backward(**change):
        a = dict(good, **dict(back, **change))
        B.op_glu_ffn_grad(a["dy"], a["x"], a["w_in"], a["w_out"], a["hidden"], a["saved"], a["dx"], a["dwi"], a["dwo"], a["ws"], act=a["act"])

    backward()
    for k in back:
        with pytest.raises(ValueError):
            backward(**{k: back[k].cpu()})
    for bad in (dict(dwi=new(2 * F, d + 8)), dict(dwo=new(d, F, dtype=torch.float32)), dict(dx=new(T, d, dtype=torch.float32))):
        with pytest.raises(ValueError):
            backward(**bad)
    for bad in (dict(act="tanh"), dict(ws=back["ws"][:-1])):
        with pytest.raises(B.SamaError):
            backward(**bad)


@pytest.mark.parametrize("dtype,T,d,F", [("bf16", 270001, 64, 8008), ("fp32", 270001, 64, 8004), ("fp32", 135001, 63, 8001)])
def test_offsets_beyond_32_bits(dtype, T, d, F):
    """More than 2^31 hidden values (the last: gates), and twice as many gates and gradients of them; checked a few thousand tokens at a time.  A sum over T tokens is
    within (T + 2) u of the sum of their sizes, which is at most the number of pieces times the bars of the pieces added up."""
    i = inputs(T, d, F, dtype, 1)
    got = run(i, "silu", dw="fp32")
    step, bars, sums = 13000, {}, {}
    for t0 in range(0, T, step):
        part = dict(i, x=i["x"][t0:t0 + step], dy=i["dy"][t0:t0 + step])
        want = exact(part, "silu")
        check({k: got[k][t0:t0 + step] for k in ("y", "hidden", "dx")}, want, dtype == "bf16")
        for k in ("dw_in", "dw_out"):
            sums[k] = want[k][0] + sums.get(k, 0.0)
            bars[k] = want[k][1] + bars.get(k, 0.0)
    check({k: got[k] for k in sums}, {k: (sums[k], bars[k] * -(-T // step)) for k in sums}, dtype == "bf16")
