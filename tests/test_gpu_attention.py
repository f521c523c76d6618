"""Attention within spans of keys, its gradients and the spans of packed documents, against plain implementations in 64 bits.

Tolerances are bounds, computed with the results, element by element.  u is 2^-24, r is what rounding to the type costs at most: 2^-8 in bf16, u in fp32 (there is none of
the probabilities there).  With a = sum |q_d k_d| scale and S the largest sum |score| + a of a row:
  a score is off by at most  e_s = (D + 8) u S  (D products in any order, the factor, the units of the exponential, the bias), capped by 2^-21 cap more in bf16, 8 u cap in fp32;
  a probability by  e_p = 2 e_s + (n + 16) u  of itself (n keys are summed; the exponential and the logarithm within 4 u), formed again from lse: by u |lse| more;
  out by  (e_p + [r in bf16]) sum p |v| + n u sum p |v| + r |out|;
  dp by  e_dp = (D + 2) u sum |do v|,  delta by  e_d = sum |do| (out's error) + D u sum |do out|, in bf16 rows of up to 8 keys by  sum (e_p' + n u) p |dp| + p e_dp;
  ds by  E = e_p' |ds| + p (e_dp + e_d) + [r |ds|] + 2^-20 p |dp - delta| where capped (1 - tanh^2),  dq by scale (sum E |k| + (n + 2) u sum |ds k|) + r |dq|, dk alike;
  dv by  (e_p' + [r]) sum p |do| + (m + 2) u sum p |do| + r |dv|   (m queries)."""
import math
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def ints(a):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32, device=DEV)


def normal(gen, *shape, dtype, std=1.0):
    return (torch.randn(*shape, device=DEV, generator=gen) * std).to(dtype)


def reference(q, k, v, spans, scale, cap, slopes, at, dout=None):
    """{name: (value, bound)} in 64 bits, [tokens, heads, width]."""
    f = torch.float64
    t = q.dtype
    r = 2.0 ** -8 if t == torch.bfloat16 else U
    soft = r if t == torch.bfloat16 else 0.0
    (Tq, Hq, D), (Tk, Hk) = q.shape, k.shape[:2]
    j = torch.arange(Tk, device=DEV)[None]
    b, e = spans[:, :1].long().clamp(min=0), spans[:, 1:].long().clamp(max=Tk)
    see = (j >= b) & (j < e)
    n = see.sum(1, keepdim=True).double()
    names = ["out", "lse"] + (["dq", "dk", "dv"] if dout is not None else [])
    shapes = dict(out=q.shape, lse=(Tq, Hq), dq=q.shape, dk=k.shape, dv=v.shape)
    val, err = ({x: torch.zeros(shapes[x], device=DEV, dtype=f) for x in names} for _ in range(2))
    zero = torch.zeros((), device=DEV, dtype=f)
    for h in range(Hq):
        g = h * Hk // Hq
        qh, kh, vh = q[:, h].double(), k[:, g].double(), v[:, g].double()
        # what is hidden takes no part, whatever it holds
        kz, vz = torch.where(see.any(0)[:, None], kh, zero), torch.where(see.any(0)[:, None], vh, zero)
        qz = torch.where(see.any(1)[:, None], qh, zero)
        s = qz @ kz.t() * scale
        size = qz.abs() @ kz.abs().t() * scale
        bend = torch.ones_like(s)
        if cap > 0:
            bend = 1 - torch.tanh(s / cap) ** 2
            s = cap * torch.tanh(s / cap)
        if slopes is not None:
            s = s - float(slopes[h]) * (at.long()[:, None] - j).abs()
        S = torch.where(see, s.abs() + size, zero).amax(1, keepdim=True)
        e_s = (D + 8) * U * S + (0.0 if cap == 0 else cap * (2.0 ** -21 if t == torch.bfloat16 else 8 * U))
        s = torch.where(see, s, torch.full_like(s, -math.inf))
        top = s.amax(1, keepdim=True)
        top = torch.where(torch.isfinite(top), top, zero)
        p = torch.exp(s - top)
        total = p.sum(1, keepdim=True)
        p = torch.where(total > 0, p / total, zero)
        e_p = 2 * e_s + (n + 16) * U
        o, o_abs = p @ vz, p @ vz.abs()
        eo = (e_p + soft + n * U) * o_abs + r * o.abs()
        val["out"][:, h], err["out"][:, h] = o, eo
        lse = torch.where(total > 0, top + torch.log(total), torch.full_like(top, -math.inf))[:, 0]
        val["lse"][:, h], err["lse"][:, h] = lse, torch.where(torch.isfinite(lse), e_p[:, 0] + 4 * U * (lse.abs() + 1), zero)
        if dout is None:
            continue
        do = torch.where(see.any(1)[:, None], dout[:, h].double(), zero)
        dp = torch.where(see, do @ vz.t(), zero)
        delta = (do * o).sum(1, keepdim=True)
        ds = p * (dp - delta) * bend
        e_dp = (D + 2) * U * (do.abs() @ vz.abs().t())
        e_d = (do.abs() * eo).sum(1, keepdim=True) + D * U * (do * o).abs().sum(1, keepdim=True)
        e_pp = e_p + U * (torch.where(torch.isfinite(lse), lse, torch.zeros_like(lse)).abs()[:, None] + 1) * 4
        if t == torch.bfloat16:
            e_d = torch.where(n <= 8, ((e_pp + n * U) * p * dp.abs() + p * e_dp).sum(1, keepdim=True), e_d)
        E = torch.where(see, e_pp * ds.abs() + p * (e_dp + e_d) + soft * ds.abs() + (2.0 ** -20 * p * (dp - delta).abs() if cap > 0 else 0.0), zero)
        val["dq"][:, h] = scale * (ds @ kz)
        err["dq"][:, h] = scale * (E @ kz.abs() + (n + 2) * U * (ds.abs() @ kz.abs())) + r * val["dq"][:, h].abs()
        m = see.sum(0)[:, None].double() * (Hq // Hk)
        val["dk"][:, g] += scale * (ds.t() @ qz)
        err["dk"][:, g] += scale * (E.t() @ qz.abs() + (m + 2) * U * (ds.abs().t() @ qz.abs()))
        val["dv"][:, g] += p.t() @ do
        err["dv"][:, g] += ((e_pp + soft) * p).t() @ do.abs() + (m + 2) * U * (p.t() @ do.abs())
    for x in ("dk", "dv"):
        if x in val:
            err[x] += r * val[x].abs()
    return {x: (val[x], err[x]) for x in names}


def close(name, got, want):
    value, bound = want
    g = got.double()
    same = (g == value) | ((g - value).abs() <= bound * (1 + 2.0 ** -10) + 1e-37)
    assert bool(same.all()), (name, float(torch.where(same, torch.zeros_like(g), (g - value).abs() - bound).abs().max()), int((~same).sum()), same.numel())


class Case:
    def __init__(self, Tq, Tk, Hq, Hk, D, t, seed=0, layout="rows", cap=0.0, slopes=False, at=None, scale=None):
        self.t, self.cap, self.scale = TYPES[t], cap, D ** -0.5 if scale is None else scale
        gen = torch.Generator(device=DEV).manual_seed(1000 * Tq + 10 * Tk + D + seed)

        def make(T, H):
            if layout == "heads":      # [heads][tokens][width]
                return normal(gen, H, T, D, dtype=self.t).transpose(0, 1)
            if layout == "wide":       # rows with something behind each head and each token
                return normal(gen, T, H + 1, D + 8, dtype=self.t)[:, :H, :D]
            return normal(gen, T, H, D, dtype=self.t)
        self.q, self.k, self.v, self.dout = make(Tq, Hq), make(Tk, Hk), make(Tk, Hk), make(Tq, Hq)
        self.dout *= 0.1
        self.make = lambda like: torch.full_like(like, 7.0)      # keeps the strides of dense layouts
        if layout == "wide":
            self.make = lambda like: torch.full((like.shape[0], like.shape[1] + 1, D + 8), 7.0, device=DEV, dtype=self.t)[:, :like.shape[1], :D]
        self.slopes = torch.exp2(-8.0 * torch.arange(1, Hq + 1, device=DEV, dtype=torch.float32) / Hq) if slopes else None
        self.at = at if at is not None else torch.arange(Tq, device=DEV, dtype=torch.int32)
        self.sizes = (Tq, Tk, Hq, Hk, D, self.t)

    def run(self, spans, grad=True):
        from paper_2310_05674_amd import binding as B
        Tq, Tk, Hq, Hk, D, t = self.sizes
        ws = torch.empty(max(B.attention_bytes(*self.sizes), B.attention_grad_bytes(*self.sizes)), dtype=torch.uint8, device=DEV).fill_(255)
        out, lse = self.make(self.q), torch.full((Tq, Hq), 7.0, device=DEV)
        kw = dict(scale=self.scale, cap=self.cap, slopes=self.slopes, at=self.at)
        B.op_attention(self.q, self.k, self.v, out, spans, ws, lse=lse, **kw)
        got = {"out": out, "lse": lse}
        if grad:
            ws.fill_(255)
            got.update(dq=self.make(self.q), dk=self.make(self.k), dv=self.make(self.v))
            B.op_attention_grad(self.dout, self.q, self.k, self.v, out, lse, spans, got["dq"], got["dk"], got["dv"], ws, **kw)
        return got

    def check(self, spans, grad=True):
        got = self.run(spans, grad)
        torch.cuda.synchronize()
        want = reference(self.q, self.k, self.v, spans, self.scale, self.cap, self.slopes, self.at, self.dout if grad else None)
        for name in want:
            close(name, got[name], want[name])
        return got


def documents(lengths, T, causal=False, prefix=None):
    """What op_attention_spans is to give."""
    spans = np.zeros((T, 2), np.int32)
    first = 0
    for n, size in enumerate(lengths):
        for i in range(first, min(first + size, T)):
            end = min(first + size, T)
            spans[i] = first, min(end, max(i + 1, first + (prefix[n] if prefix is not None else 0))) if causal else end
        first += size
    return spans


@pytest.mark.parametrize("lengths,T,causal,prefix", [([5], 5, False, None), ([1], 1, True, None), ([3, 0, 4], 9, True, None), ([3, 0, 4], 9, False, None), ([10, 300, 1, 77], 400, True, [3, 100, 5, 0]),
                                                     ([10, 300, 1, 77], 350, True, [3, 1000, 5, 0]), ([], 4, True, None), ([600, 423], 1023, False, [1, 2])])
def test_spans(lengths, T, causal, prefix):
    from paper_2310_05674_amd import binding as B
    offsets = ints(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32))
    spans = torch.full((T, 2), 9, dtype=torch.int32, device=DEV)
    B.op_attention_spans(offsets, spans, causal=causal, prefix=None if prefix is None else ints(np.asarray(prefix, np.int32)))
    want = documents(lengths, T, causal, prefix)
    got = spans.cpu().numpy()
    some = want[:, 0] < want[:, 1]
    assert np.array_equal(got[some], want[some]) and np.all(got[~some] == 0)


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("T,Hq,Hk,D", [(1, 1, 1, 8), (2, 2, 1, 64), (31, 2, 2, 128), (32, 1, 1, 64), (33, 3, 1, 40), (65, 4, 2, 128), (129, 2, 1, 96), (300, 6, 2, 64), (700, 4, 4, 32), (1025, 2, 2, 128)])
@pytest.mark.parametrize("causal", [False, True])
def test_one_document(T, Hq, Hk, D, causal, t):
    Case(T, T, Hq, Hk, D, t).check(ints(documents([T], T, causal)))


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("T,D", [(2180, 64), (2180, 128), (2700, 64), (4100, 64), (4100, 128), (8200, 64)])
def test_many_workgroups(T, D, t):
    """Rows and keys for workgroups of 32, 64 and 128 of them, forward and backward."""
    Case(T, T, 16, 16, D, t).check(ints(documents([T * 2 // 3, 37, T // 4], T, True)))


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("cap,slopes", [(20.0, False), (0.0, True), (5.0, True)])
@pytest.mark.parametrize("T,D", [(2700, 64), (2700, 128), (4100, 64), (4100, 128)])
def test_many_workgroups_capped_and_biased(T, D, cap, slopes, t):
    Case(T, T, 16, 16, D, t, cap=cap, slopes=slopes).check(ints(documents([T * 2 // 3, 37, T // 4], T, True, [700, 20, 1])))


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("cap,slopes", [(20.0, False), (0.0, True), (5.0, True)])
@pytest.mark.parametrize("T,D", [(90, 64), (333, 128)])
def test_capped_and_biased(T, D, cap, slopes, t):
    Case(T, T, 4, 2, D, t, cap=cap, slopes=slopes).check(ints(documents([T // 3, T // 2], T, True, [T // 6, 5])))


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("G", [3, 5, 7, 8, 64])
def test_shared_key_heads(G, t):
    Case(77, 77, 2 * G, 2, 64, t).check(ints(documents([50, 20], 77, True)))


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", ["heads", "wide"])
def test_layouts(layout, t):
    c = Case(150, 150, 4, 2, 80, t, layout=layout)
    got = c.check(ints(documents([100, 41], 150, True)))
    if layout == "wide":                                   # nothing beside the rows
        for x in ("out", "dq", "dk", "dv"):
            whole = got[x]._base if got[x]._base is not None else got[x]
            assert bool((whole[:, -1] == 7).all()) and bool((whole[:, :, 80:] == 7).all())


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("T,Hk", [(300, 2), (2200, 16), (2700, 16), (4230, 16)])
def test_spans_in_any_order(T, Hk, t):
    """Spans that overlap, lie apart, are empty, single, turned round or reach over the ends, in no order."""
    r = np.random.RandomState(3)
    a, n = r.randint(-5, T, T), r.choice([0, 1, 1, 2, 31, 64, 100, T + 9], T)
    spans = np.stack([a, a + n], 1)
    spans[7], spans[11], spans[12] = (50, 20), (-2 ** 31, 2 ** 31 - 1), (T - 1, 2 ** 31 - 1)
    Case(T, T, Hk, Hk, 64, t).check(ints(spans))


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("n,lengths", [(1, [1]), (1, [5000]), (3, [700, 1, 2049]), (32, [97] * 32)])
@pytest.mark.parametrize("D,G", [(128, 4), (64, 1), (40, 3)])
def test_new_tokens_over_caches(n, lengths, D, G, t):
    room = [x // 64 * 64 + 64 for x in lengths]
    first = np.concatenate([[0], np.cumsum(room)])
    spans = np.stack([first[:-1], first[:-1] + lengths], 1)
    at = ints(spans[:, 1] - 1)
    c = Case(n, int(first[-1]), 2 * G, 2, D, t, slopes=True, at=at)
    for i in range(n):                                     # what a cache has no token for yet
        c.k[int(spans[i, 1]):int(first[i + 1])] = float("nan")
        c.v[int(spans[i, 1]):int(first[i + 1])] = float("inf")
    c.check(ints(spans))


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("T,H", [(100, 2), (2180, 16), (2700, 16), (4100, 16)])
def test_what_is_hidden_may_hold_anything(T, H, t):
    """Rows of padding between documents, of all inputs, hold NaN and infinity."""
    c = Case(T, T, H, H, 64, t)
    spans = np.zeros((T, 2), np.int32)
    for a, b in ((3, 20), (24, 60), (61, T - 7)):
        for i in range(a, b):
            spans[i] = a, i + 1
    empty = torch.as_tensor(spans[:, 0] == spans[:, 1], device=DEV)
    for x, y in ((c.q, float("nan")), (c.k, float("inf")), (c.v, float("nan")), (c.dout, -float("inf"))):
        x[empty] = y
    got = c.check(ints(spans))
    for x in ("out", "dq", "dk", "dv"):
        assert bool((got[x][empty] == 0).all())


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [96, 1100])
def test_what_is_not_finite_reaches_whom_sees_it(T, t):
    """A later token's NaN in k and v stays with the queries behind it, and its column of v with that column."""
    c = Case(T, T, 1, 1, 64, t)
    spans = ints(documents([T], T, True))
    clean = c.run(spans)
    at = T - 40
    v0 = c.v.clone()
    c.v[at, 0, 5] = float("inf")
    got = c.run(spans)
    assert torch.equal(got["out"][:at], clean["out"][:at]) and torch.equal(got["dq"][:at], clean["dq"][:at])
    bad = ~torch.isfinite(got["out"][:, 0])
    assert bool(bad[at:, 5].all()) and int(bad.sum()) == T - at
    c.v.copy_(v0)
    c.k[at, 0, 9] = float("nan")
    got = c.run(spans)
    assert torch.equal(got["out"][:at], clean["out"][:at]) and torch.equal(got["dq"][:at], clean["dq"][:at])
    assert bool(torch.isnan(got["out"][at:]).all()) and bool(torch.isnan(got["dq"][at:]).all())
    c.k.copy_(torch.nan_to_num(c.k))
    c.k[at, 0, 9] = 0.5
    clean = c.run(spans)
    c.dout[3] = float("nan")                               # sees the first four keys
    got = c.run(spans)
    for x in ("dk", "dv"):
        assert torch.equal(got[x][4:], clean[x][4:]) and not bool(torch.isfinite(got[x][:4]).any())


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("cap,slopes", [(0.0, False), (5.0, True)])
@pytest.mark.parametrize("n", [1, 2, 3, 5, 8, 9])
def test_few_keys(n, cap, slopes, t):
    """Rows of a few keys, beside each other in a group."""
    T = 100
    first = np.arange(T) // n * n
    Case(T, T, 6, 2, 80, t, cap=cap, slopes=slopes).check(ints(np.stack([first, np.minimum(first + n, T)], 1)))


@pytest.mark.parametrize("t", ["bf16", "fp32"])
def test_far_rows(t):
    """Keys and values, their gradients and the queries in rows 2^17 values apart: offsets pass 2^31 values, and 2^33 bytes in fp32."""
    Tq, Tk, D, ld = 40, 20011, 64, 2 ** 17
    c = Case(Tq, Tk, 2, 1, D, t, at=torch.arange(Tq, device=DEV, dtype=torch.int32) + (Tk - Tq), slopes=True)
    room = torch.empty(Tk, ld, dtype=c.t, device=DEV)
    places = [room[:, 64 * i:64 * i + 64].view(Tk, 1, D) for i in range(4)]
    far = torch.empty(Tq, 2, 2 ** 21 // 2, dtype=c.t, device=DEV)[:, :, :D]
    for i, x in enumerate(("k", "v")):
        places[i].copy_(getattr(c, x))
        setattr(c, x, places[i])
    c.q = far.copy_(c.q)
    plain, used = c.make, []

    def make(like):
        if like.shape[0] == Tq:
            return plain(like)
        used.append(places[2 + len(used)].fill_(7.0))
        return used[-1]
    c.make = make
    b = np.array([0, 5, 19000, 20010] * 10)
    c.check(ints(np.stack([b, np.minimum(b + [20011, 1, 900, 1] * 10, Tk)], 1)))
    assert len(used) == 2


def test_no_queries_and_no_keys():
    from paper_2310_05674_amd import binding as B
    new = lambda *s, dtype=torch.bfloat16: torch.full(s, 7, dtype=dtype, device=DEV)
    ws = new(4096, dtype=torch.uint8)
    q, out, lse, spans = new(5, 4, 64), new(5, 4, 64), new(5, 4, dtype=torch.float32), ints(np.array([[0, 9]] * 5))
    none = new(0, 2, 64)
    B.op_attention(q, none, none, out, spans, ws, lse=lse)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    dq = new(5, 4, 64)
    B.op_attention_grad(q, q, none, none, out, lse, spans, dq, none, none, ws)
    assert bool((dq == 0).all())
    k, dk, dv = new(300, 2, 64), new(300, 2, 64), new(300, 2, 64)
    q = new(0, 4, 64)
    B.op_attention(q, k, k, q, spans[:0], ws, lse=lse[:0])
    B.op_attention_grad(q, q, k, k, q, lse[:0], spans[:0], q, dk, dv, ws)
    assert bool((dk == 0).all()) and bool((dv == 0).all())


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("Tq,Tk,Hq,Hk,D", [(700, 700, 4, 2, 64), (2200, 2200, 8, 8, 128), (4200, 4200, 16, 16, 64), (2, 9000, 8, 2, 128)])
def test_the_same_call_gives_the_same_bits(Tq, Tk, Hq, Hk, D, t):
    c = Case(Tq, Tk, Hq, Hk, D, t, slopes=True)
    spans = ints(np.stack([np.arange(Tq) // 500 * 500, np.arange(Tq) + (Tk - Tq) + 1], 1))
    first = c.run(spans)
    for _ in range(3):
        got = c.run(spans)
        for x in first:
            assert torch.equal(got[x], first[x]), x


def test_gradients_against_differences():
    """Gradients along a direction of q, k and v against central differences of sum(dout out), formed in 64 bits by reference() at steps h and 2 h: truncation is
    a third of what the two differ by; the sums, of 10^4 values up to 1, round by less than 1e-10.  The formula's gradients keep within that, the kernel's within their bounds
    more, added up along the direction."""
    T, Hq, Hk, D, cap = 70, 4, 2, 40, 8.0
    c = Case(T, T, Hq, Hk, D, "fp32", cap=cap, slopes=True)
    spans = ints(documents([33, 30], T, True, [9, 0]))
    got = c.run(spans)
    want = reference(c.q, c.k, c.v, spans, c.scale, cap, c.slopes, c.at, c.dout)
    gen = torch.Generator(device=DEV).manual_seed(5)
    for x in ("q", "k", "v"):
        way = torch.randn(getattr(c, x).shape, device=DEV, generator=gen, dtype=torch.float64)

        def loss(h):
            moved = {y: getattr(c, y).double() for y in ("q", "k", "v")}
            moved[x] = moved[x] + h * way
            return float((reference(moved["q"], moved["k"], moved["v"], spans, c.scale, cap, c.slopes, c.at)["out"][0] * c.dout.double()).sum())
        h = 2.0 ** -12
        one, two = ((loss(s) - loss(-s)) / (2 * s) for s in (h, 2 * h))
        tolerance = abs(one - two) + 1e-10 / h
        value, bound = want["d" + x]
        assert abs(float((value * way).sum()) - one) <= tolerance < 1e-4
        assert abs(float((got["d" + x].double() * way).sum()) - one) <= tolerance + float((bound * way.abs()).sum())


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("Tk,H", [(1000, 2), (12000, 2), (40000, 1), (12000, 60)])   # keys in one part, and split
def test_what_is_not_finite_reaches_a_query_far_away(Tk, H, t):
    """Values of keys so far behind that their probability is zero in 32 bits: zero times what is not finite is not finite, in whichever part of the keys it lies."""
    from paper_2310_05674_amd import binding as B
    D = 64
    gen = torch.Generator(device=DEV).manual_seed(Tk + H)
    q, k, v = (normal(gen, n, H, D, dtype=TYPES[t]) for n in (2, Tk, Tk))
    spans, at = ints(np.array([[0, Tk], [Tk // 2, Tk]])), ints([Tk - 1, Tk - 1])
    slopes = torch.ones(H, device=DEV)
    ws = torch.empty(B.attention_bytes(2, Tk, H, H, D, TYPES[t]), dtype=torch.uint8, device=DEV)

    def run():
        out, lse = torch.full_like(q, 7.0), torch.full((2, H), 7.0, device=DEV)
        ws.fill_(255)
        B.op_attention(q, k, v, out, spans, ws, slopes=slopes, at=at, lse=lse)
        return out, lse
    clean, clean_lse = run()
    assert bool(torch.isfinite(clean).all())
    for value in (float("nan"), math.inf, -math.inf):
        kept = v[3, :, 9].clone()
        v[3, :, 9] = value                                    # only the first query sees it
        out, lse = run()
        v[3, :, 9] = kept
        assert torch.equal(out[1], clean[1]) and torch.equal(lse, clean_lse)
        assert not bool(torch.isfinite(out[0, :, 9]).any())
        rest = torch.arange(D, device=DEV) != 9
        assert torch.equal(out[0][:, rest], clean[0][:, rest])


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("T,H", [(100, 2), (2180, 16), (4100, 16)])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_of_minus_infinity_alone(T, H, D, t):
    """The softmax of scores that are all minus infinity is no number: neither is out, nor what the query's gradients reach.  One score that is finite is enough for out, and who sees
    nothing of it keeps his bits."""
    c = Case(T, T, H, H, D, t)
    third = T // 3
    spans = documents([third, third, third], T, True)
    c.q[:, :, 0], c.k[:, :, 0] = 1.0, 0.5
    clean = c.run(ints(spans))
    c.k[:third, :, 0] = -math.inf                             # of the first document all, of the second all but its first
    c.k[third + 1:2 * third, :, 0] = -math.inf
    got = c.run(ints(spans))
    assert bool(torch.isnan(got["out"][:third]).all()) and bool((got["lse"][:third] == -math.inf).all())
    for x in ("dq", "dk", "dv"):
        assert not bool(torch.isfinite(got[x][:third]).all(-1).any()), x
    first = c.v[third].double()                               # probability 1, within 64 u for a score of up to 40
    assert bool(((got["out"][third:2 * third].double() - first).abs() <= ((2.0 ** -8 if t == "bf16" else U) + 64 * U) * first.abs()).all()) and bool(torch.isfinite(got["lse"][third:2 * third]).all())
    for x in clean:
        assert torch.equal(got[x][2 * third:], clean[x][2 * third:]), x


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_of_minus_infinity_in_split_keys(D, t):
    """The same for few queries over keys that are split: all scores minus infinity, all of some parts, no key, no key in some parts."""
    Tk = 9000
    c = Case(4, Tk, 2, 2, D, t, at=ints([Tk - 1] * 4))
    c.q[:, :, 0], c.k[:, :, 0] = 1.0, 0.5
    spans = np.array([[0, 5000], [0, Tk], [17, 17], [5000, Tk]])
    c.k[:5000, :, 0] = -math.inf
    got = c.run(ints(spans), grad=False)
    assert bool(torch.isnan(got["out"][0]).all()) and bool((got["lse"][0] == -math.inf).all())
    assert bool((got["out"][2] == 0).all()) and bool((got["lse"][2] == -math.inf).all())
    c.k[:5000, :, 0] = 0.5
    want = reference(c.q, c.k, c.v, ints(spans[3:].repeat(4, 0)), c.scale, 0.0, None, c.at)
    for x in ("out", "lse"):
        close(x, got[x][1::2], (want[x][0][1::2], want[x][1][1::2]))


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("Tk", [700, 16640])
def test_one_query_out_of_a_long_text(Tk, t):
    """[heads][tokens][width] memory: a query's heads lie a whole text apart, and it is the only token of its call."""
    D, i = 128, Tk - 100
    c = Case(Tk, Tk, 2, 2, D, t, layout="heads")
    new, c.at = c.q, ints([i])
    c.q, c.dout, c.sizes = new[i:i + 1], c.dout[i:i + 1], (1, Tk, 2, 2, D, c.t)
    whole = [torch.full((2, Tk, D), 7.0, dtype=c.t, device=DEV) for _ in range(2)]
    places = [w.transpose(0, 1)[i:i + 1] for w in whole]
    plain = c.make
    c.make = lambda like: places.pop() if like.shape[0] == 1 else plain(like)
    c.check(ints(np.array([[3, i + 1]])))
    for w in whole:                                        # nothing beside the token
        assert bool((w[:, :i] == 7).all()) and bool((w[:, i + 1:] == 7).all()) and not bool((w[:, i] == 7).all())


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [8, 72])
def test_as_many_key_heads_as_there_may_be(D, t):
    """2^20 key heads of one token, the most workgroups for a few rows.  A single key has probability 1, within 2 e_s + 17 u (e_s above, S at most 2 sum |q k| scale) where it is formed from
    the logarithm again: out = v, dv = dout, dq = dk = 0."""
    H = 2 ** 20
    c = Case(1, 1, H, H, D, t)
    got = c.run(ints(np.array([[0, 1]])))
    size = (c.q.float().abs() * c.k.float().abs()).sum(-1, keepdim=True) * c.scale
    for name, want in (("out", c.v), ("dv", c.dout)):
        off = 2 * (D + 8) * U * 2 * size + (17 + 8) * U + (2.0 ** -8 + 2.0 ** -8 if t == "bf16" else U)
        assert bool(((got[name].float() - want.float()).abs() <= off * want.float().abs()).all()), name
    s = (c.q.double() * c.k.double()).sum(-1) * c.scale
    assert bool(((got["lse"].double() - s).abs() <= (2 * (D + 8) * U * 2 * size[..., 0] + 21 * U * (s.abs() + 1))).all())
    assert bool((got["dq"] == 0).all()) and bool((got["dk"] == 0).all())


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hk,G", [(1, 1), (2, 33), (5, 8), (33, 1), (100, 2), (130, 1), (200, 1), (256, 1)])
def test_keys_in_one_round_of_parts_and_in_two(Hk, G, D, t):
    """Two new tokens over caches, with as many key heads as make parts of every number, and one that sees keys of a few parts alone."""
    Tk = 8001
    Case(3, Tk, G * Hk, Hk, D, t, at=ints([2999, Tk - 1, 7000])).check(ints([[0, 3000], [3000, Tk], [6990, 7001]]), grad=False)


class ProductCase(Case):
    """Queries, keys and values, and their gradients, as parts of one product's rows."""
    def __init__(self, T, Hq, Hk, D, t, **kw):
        super().__init__(T, T, Hq, Hk, D, t, **kw)
        rows, self.grads = torch.cat([self.q, self.k, self.v], 1), torch.full((T, Hq + 2 * Hk, D), 7.0, device=DEV, dtype=self.t)
        self.q, self.k, self.v = rows.split([Hq, Hk, Hk], 1)
        plain, self.made = self.make, 0

        def make(like):      # out, then dq, dk, dv
            self.made += 1
            return plain(like) if self.made % 4 == 1 else self.grads.split([Hq, Hk, Hk], 1)[(self.made - 2) % 4]
        self.make = make


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("T,Hk,G,D", [(2180, 4, 4, 72), (4100, 8, 3, 80), (8200, 8, 2, 96), (6200, 8, 5, 128), (8200, 16, 2, 64), (4100, 8, 7, 40)])
def test_many_workgroups_of_shared_key_heads(T, Hk, G, D, t):
    """Shared key heads, and widths that leave pieces of a tile empty, in workgroups of every size, with documents of every kind and tokens outside them."""
    ProductCase(T, G * Hk, Hk, D, t).check(ints(documents([T * 2 // 3, 0, 37, T // 4, 1], T, True, [300, 0, 20, 1, 0])))


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("T,Hk,G,D", [(4100, 8, 3, 80), (8200, 8, 2, 96), (8200, 16, 2, 48)])
def test_many_workgroups_of_shared_key_heads_capped_and_biased(T, Hk, G, D, t):
    ProductCase(T, G * Hk, Hk, D, t, cap=5.0, slopes=True).check(ints(documents([T // 2, 500, T // 4], T, True)))


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("T,Hk,G,D", [(300, 2, 3, 128), (2180, 8, 2, 128), (4100, 8, 2, 96), (8200, 8, 2, 128), (8200, 16, 2, 64)])
def test_what_is_hidden_and_what_is_seen_in_workgroups_of_every_size(T, Hk, G, D, t):
    """Padding that holds NaN and infinity changes no bit; a key, value or gradient that is not finite changes whom it reaches and nobody else."""
    c = ProductCase(T, G * Hk, Hk, D, t)
    spans = documents([T // 2 + 3], T, True)
    tail = slice(T // 2 + 11, T - 5)
    spans[tail] = [[T // 2 + 11, i + 1] for i in range(tail.start, tail.stop)]
    empty = torch.as_tensor(spans[:, 0] == spans[:, 1], device=DEV)
    spans = ints(spans)

    def run():
        c.grads.fill_(7.0)
        return {x: v.clone() for x, v in c.run(spans).items()}
    clean = run()
    for x, y in ((c.q, float("nan")), (c.k, math.inf), (c.v, float("nan")), (c.dout, -math.inf)):
        x[empty] = y
    got = run()
    for x in ("out", "dq", "dk", "dv"):
        assert torch.equal(got[x][~empty], clean[x][~empty]) and bool((got[x][empty] == 0).all()), x
    at = T // 4                                            # a token of the first document, seen from itself on
    kept = c.v[at, 0, 5].clone()
    c.v[at, 0, 5] = math.inf
    got = run()
    c.v[at, 0, 5] = kept
    reached = slice(at, T // 2 + 3)
    bad = ~torch.isfinite(got["out"])
    assert bool(bad[reached, :G, 5].all()) and int(bad.sum()) == (reached.stop - at) * G
    for x in ("out", "dq"):
        assert torch.equal(got[x][:at], clean[x][:at]) and torch.equal(got[x][tail], clean[x][tail]) and torch.equal(got[x][:, G:], clean[x][:, G:]), x
    for x in ("dk", "dv"):
        assert torch.equal(got[x][:, 1:], clean[x][:, 1:]) and torch.equal(got[x][tail], clean[x][tail]), x
    kept = c.dout[at, 0].clone()
    c.dout[at, 0] = float("nan")                           # sees the keys up to its own
    got = run()
    c.dout[at, 0] = kept
    for x in ("dk", "dv"):
        assert not bool(torch.isfinite(got[x][:at + 1, 0]).any()) and torch.equal(got[x][at + 1:], clean[x][at + 1:]) and torch.equal(got[x][:, 1:], clean[x][:, 1:]), x
    rest = torch.ones(T, G * Hk, dtype=torch.bool, device=DEV)
    rest[at, 0] = False
    assert not bool(torch.isfinite(got["dq"][at, 0]).any()) and torch.equal(got["dq"][rest], clean["dq"][rest])
