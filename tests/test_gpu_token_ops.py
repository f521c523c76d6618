"""The operators of a token model's step against plain implementations in 64 bits.

Tolerances.  u = 2^-24 is the unit roundoff of fp32, 2^-8 that of bf16.  A lookup is one fp32 product and one rounding: exact.  A sum of c
fp32 terms in any order is within c u of the sum of their sizes; the scaling and the store add one rounding each."""
import numpy as np
import pytest
import torch
from datagen import CounterRNG

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32, U16 = 2.0 ** -24, 2.0 ** -8
T = {"fp32": torch.float32, "bf16": torch.bfloat16}


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def values(seed, *shape):
    return torch.as_tensor(CounterRNG(seed).normal(1, int(np.prod(shape))).reshape(shape).astype(np.float32), device=DEV)


def token_ids(kind, n, V, seed):
    r = np.random.RandomState(seed)
    if kind == "same":
        a = np.full(n, V // 3)
    elif kind == "zipf":
        a = np.minimum((r.zipf(1.2, n) - 1), V - 1)
    elif kind == "distinct":
        a = r.permutation(max(n, V))[:n] % V
    elif kind == "outside":
        a = r.randint(-3, V + 3, n)
    else:   # runs
        a = np.repeat(r.randint(0, V, n // 7 + 1), 7)[:n]
    return torch.as_tensor(a.astype(np.int32), device=DEV)


def rows(shape, dtype, ld, offset):
    """An uninitialised [n, d] view with row stride ld that begins `offset` values into its memory, over a buffer of ones."""
    n, d = shape
    whole = torch.ones(offset + max(n, 1) * ld, dtype=dtype, device=DEV)
    return whole[offset:offset + n * ld].view(n, ld)[:, :d], whole


# ------------------------------------------------------------------------------------------------------ lookup
@pytest.mark.parametrize("table_t,out_t", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "fp32"), ("bf16", "bf16")])
@pytest.mark.parametrize("n,V,d", [(1, 1, 1), (3, 10, 7), (128, 300, 64), (703, 1000, 100), (4097, 8192, 256), (37, 50, 1030), (2051, 600, 768), (9, 12, 2048)])
def test_lookup(n, V, d, table_t, out_t):
    from paper_2310_05674_amd import binding as B
    table = values(n + d, V, d).to(T[table_t])
    ids = token_ids("outside", n, V, n)
    out = torch.empty(n, d, dtype=T[out_t], device=DEV)
    B.op_embedding(table, ids, out, scale=1.7)
    want = (table.float()[ids.clamp(0, V - 1).long()] * torch.tensor(1.7, device=DEV)).to(T[out_t])
    assert torch.equal(out, want)


@pytest.mark.parametrize("ldt,ldo,offset", [(72, 64, 0), (64, 80, 8), (65, 64, 0), (64, 67, 0), (64, 64, 1), (64, 64, 4)])
def test_lookup_strides(ldt, ldo, offset):
    from paper_2310_05674_amd import binding as B
    for table_t, out_t in (("fp32", "bf16"), ("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")):
        table, _ = rows((33, 64), T[table_t], ldt, offset)
        table.copy_(values(3, 33, 64))
        out, whole = rows((50, 64), T[out_t], ldo, offset)
        ids = token_ids("zipf", 50, 33, 1)
        B.op_embedding(table, ids, out, scale=0.5)
        assert torch.equal(out, (table.float()[ids.long()] * 0.5).to(T[out_t]))
        kept = torch.ones_like(whole)
        kept[offset:offset + 50 * ldo].view(50, ldo)[:, :64] = out
        assert torch.equal(whole, kept)                       # nothing beside the rows


def test_lookup_padding_and_unusual_values():
    from paper_2310_05674_amd import binding as B
    table = values(1, 20, 96)
    table[4] = float("nan"); table[5, 3] = float("inf"); table[6] = torch.finfo(torch.float32).tiny
    ids = torch.tensor([4, 5, 4, 6, -1, 25, 0, 4], dtype=torch.int32, device=DEV)
    for out_t in ("fp32", "bf16"):
        out = torch.empty(8, 96, dtype=T[out_t], device=DEV)
        B.op_embedding(table, ids, out, scale=2.0, pad_id=4)
        want = (table[ids.clamp(0, 19).long()] * 2.0).to(T[out_t])
        want[ids == 4] = 0
        assert torch.equal(out, want)
        B.op_embedding(table, ids, out, scale=2.0, pad_id=19)   # 25 is not the padding: padding is a token's own id, not what it is clamped to
        assert torch.equal(out[5], (table[19] * 2.0).to(T[out_t])) and bool(torch.isnan(out[0].float()).all())
    empty = torch.empty(0, 96, device=DEV)
    B.op_embedding(table, ids[:0], empty)


# ------------------------------------------------------------------------------------------------------ gradient
def check_grad(dy, ids, V, got, scale, pad=-1, start=None):
    i = ids.cpu().numpy()
    real = i != pad if pad >= 0 else np.ones(len(i), bool)
    v = np.clip(i, 0, V - 1)[real]
    x = f64(dy)[real] * scale
    want, size = np.zeros((V, dy.shape[1])), np.zeros((V, dy.shape[1]))
    np.add.at(want, v, x); np.add.at(size, v, np.abs(x))
    if start is not None:
        want += start; size += np.abs(start)
    count = np.bincount(v, minlength=V)[:, None].astype(np.float64)
    tol = (count + 3) * U32 * size + (U16 * np.abs(want) * (1 + 1e-3) if got.dtype == torch.bfloat16 else 0.0)
    g = f64(got)
    assert np.all(np.abs(g - want) <= tol + 1e-40), float(np.max(np.abs(g - want) - tol))
    if start is None:
        assert np.all(g[count[:, 0] == 0] == 0.0)


def grad_of(dy, ids, V, grad_t, **kw):
    from paper_2310_05674_amd import binding as B
    n, d = dy.shape
    ws = torch.full((B.embedding_grad_bytes(n, V, d),), 0xa5, dtype=torch.uint8, device=DEV)   # nothing is expected in it
    grad = torch.full((V, d), 7.0, dtype=T[grad_t], device=DEV)
    B.op_embedding_grad(dy, ids, grad, ws, **kw)
    return grad


@pytest.mark.parametrize("dy_t,grad_t", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "fp32"), ("bf16", "bf16")])
@pytest.mark.parametrize("kind,n,V,d", [("zipf", 1, 1, 1), ("zipf", 2, 5, 3), ("runs", 63, 7, 64), ("same", 64, 512, 72), ("zipf", 65, 513, 100), ("outside", 703, 1000, 256),
                                        ("same", 1000, 3, 520), ("zipf", 4096, 8192, 768), ("distinct", 4096, 5000, 64), ("runs", 5000, 40, 264), ("zipf", 1500, 300000, 8)])
def test_token_gradient(kind, n, V, d, dy_t, grad_t):
    dy = values(n + V, n, d).to(T[dy_t])
    ids = token_ids(kind, n, V, n + d)
    got = grad_of(dy, ids, V, grad_t, scale=1.25)
    check_grad(dy, ids, V, got, 1.25)
    assert torch.equal(got, grad_of(dy, ids, V, grad_t, scale=1.25))      # a fixed order


@pytest.mark.parametrize("kind,n,d,dy_t", [("same", 70001, 64, "bf16"), ("zipf", 70001, 136, "bf16"), ("runs", 40000, 264, "fp32"), ("same", 33000, 20, "fp32"), ("zipf", 300000, 16, "fp32")])
def test_token_gradient_long_runs(kind, n, d, dy_t):
    """Runs over many workgroups, and every number of sorted rows that a wave may take."""
    dy = values(n, n, d).to(T[dy_t])
    ids = token_ids(kind, n, 1000, 5)
    got = grad_of(dy, ids, 1000, "fp32", scale=1.0)
    check_grad(dy, ids, 1000, got, 1.0)
    assert torch.equal(got, grad_of(dy, ids, 1000, "fp32", scale=1.0))


def test_token_gradient_every_row_count():
    """Chunk borders: 1 to 70 rows and around the sizes where a workgroup, and a wave's share, changes."""
    for n in list(range(1, 71)) + [127, 128, 129, 255, 256, 257, 511, 513, 4095, 4097, 8191, 8193]:
        dy = values(n, n, 24)
        for kind in ("runs", "same"):
            ids = token_ids(kind, n, 9, n)
            check_grad(dy, ids, 9, grad_of(dy, ids, 9, "fp32", scale=1.0), 1.0)


def test_token_gradient_padding():
    n, V, d = 3000, 900, 128
    dy, ids = values(1, n, d), token_ids("zipf", n, V, 2)
    ids[::3] = 0
    dy[ids == 0] = float("nan")                                        # rows of padding are not read
    check_grad(torch.nan_to_num(dy), ids, V, grad_of(dy, ids, V, "fp32", scale=2.0, pad_id=0), 2.0, pad=0)
    ids.fill_(5)
    assert not grad_of(dy, ids, V, "fp32", pad_id=5).any()             # nothing but padding
    assert not grad_of(dy[:0], ids[:0], V, "fp32").any()               # no token


@pytest.mark.parametrize("ldy,ldg,offset", [(80, 64, 0), (64, 96, 4), (67, 64, 0), (64, 65, 0), (64, 64, 1)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_token_gradient_strides_and_accumulation(ldy, ldg, offset, accumulate):
    from paper_2310_05674_amd import binding as B
    n, V, d = 900, 200, 64
    for dy_t, grad_t in (("fp32", "fp32"), ("bf16", "fp32"), ("bf16", "bf16")):
        dy, _ = rows((n, d), T[dy_t], ldy, offset)
        dy.copy_(values(4, n, d))
        ids = token_ids("zipf", n, V // 2, 3)
        grad, whole = rows((V, d), T[grad_t], ldg, offset)
        grad.copy_(values(5, V, d))
        before = f64(grad)
        ws = torch.empty(B.embedding_grad_bytes(n, V, d), dtype=torch.uint8, device=DEV)
        B.op_embedding_grad(dy, ids, grad, ws, scale=0.75, accumulate=accumulate)
        check_grad(dy, ids, V, grad, 0.75, start=before if accumulate else None)
        kept = torch.ones_like(whole)
        kept[offset:offset + V * ldg].view(V, ldg)[:, :d] = grad
        assert torch.equal(whole, kept)
        if accumulate:
            unseen = np.setdiff1d(np.arange(V), ids.cpu().numpy())
            assert np.array_equal(f64(grad)[unseen], before[unseen])


def test_token_gradient_is_the_lookups_derivative():
    """<dy, lookup(W + e E) - lookup(W - e E)> / 2 e = <grad, E> for a lookup that is linear: only roundings differ."""
    from paper_2310_05674_amd import binding as B
    n, V, d, scale, e = 500, 300, 72, 1.5, 0.25
    W, E, dy = values(1, V, d), values(2, V, d), values(3, n, d)
    ids = token_ids("zipf", n, V, 4)
    grad = grad_of(dy, ids, V, "fp32", scale=scale, pad_id=1)
    up, down = torch.empty(n, d, device=DEV), torch.empty(n, d, device=DEV)
    B.op_embedding(W + e * E, ids, up, scale=scale, pad_id=1)
    B.op_embedding(W - e * E, ids, down, scale=scale, pad_id=1)
    terms = f64(dy) * (f64(up) - f64(down)) / (2 * e)
    # up and down carry three roundings each (e E, the sum, the product) of values of size |W| + |e E|
    tol = np.sum(np.abs(f64(dy)) * 6 * U32 * (np.abs(f64(up)) + np.abs(f64(down))) / (2 * e)) + n * U32 * np.sum(np.abs(f64(grad) * f64(E)))
    assert abs(terms.sum() - np.sum(f64(grad) * f64(E))) <= tol


def test_token_ops_in_a_graph_and_on_another_stream():
    from paper_2310_05674_amd import binding as B
    n, V, d = 2500, 4000, 192
    table, dy, ids = values(1, V, d), values(2, n, d), token_ids("zipf", n, V, 3)
    out, grad = torch.empty(n, d, device=DEV), torch.empty(V, d, device=DEV)
    ws = torch.empty(B.embedding_grad_bytes(n, V, d), dtype=torch.uint8, device=DEV)
    cws, norm = torch.empty(B.grad_clip_bytes(), dtype=torch.uint8, device=DEV), torch.empty(2, device=DEV)
    flat = torch.empty(V * d, device=DEV)

    def step():
        B.op_embedding(table, ids, out, scale=3.0)
        B.op_embedding_grad(dy, ids, grad, ws, scale=3.0)
        B.op_grad_clip([grad], 1.0, norm, cws, out=flat)

    step()
    want = [t.clone() for t in (out, grad, norm, flat)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t in (out, grad, norm, flat):
            t.fill_(9.0)
        step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((out, grad, norm, flat), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        dy.copy_(values(20 + k, n, d)); ids.copy_(token_ids("zipf", n, V, 30 + k))
        step()
        want = [t.clone() for t in (out, grad, norm, flat)]
        for t in (out, grad, norm, flat):
            t.fill_(9.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, grad, norm, flat), want)), k


# ------------------------------------------------------------------------------------------------------ clipping
def clip(grads, max_norm, out=None, status=None):
    from paper_2310_05674_amd import binding as B
    ws = torch.full((B.grad_clip_bytes(),), 0xff, dtype=torch.uint8, device=DEV)
    norm = torch.full((2,), -1.0, device=DEV)
    B.op_grad_clip(grads, max_norm, norm, ws, out=out, status=status)
    return norm.cpu().numpy().astype(np.float64)


def gradients(sizes, seed, types):
    out = []
    for k, n in enumerate(sizes):
        t = T[types[k % len(types)]]
        out.append((values(seed + k, max(n, 1))[:n] * 10.0 ** -(k % 3)).to(t))
    return out


@pytest.mark.parametrize("types", [("fp32",), ("bf16",), ("bf16", "fp32")])
@pytest.mark.parametrize("sizes", [(1,), (0, 5, 0), (7, 8, 9), (8191, 8192, 8193, 8200), (100003, 1, 64), tuple(range(300)), (2 ** 21 + 5, 3)])
@pytest.mark.parametrize("max_norm", [0.5, 1e9])
def test_clipping(sizes, types, max_norm):
    grads = gradients(sizes, 11, types)
    before = [f64(g) for g in grads]
    norm = np.sqrt(sum(float(np.sum(b * b)) for b in before))
    factor = min(1.0, max_norm / (norm + 1e-6))
    total = sum(sizes)
    out = torch.full((total,), 3.0, device=DEV)
    kept = [g.clone() for g in grads]
    status = torch.full((1,), 5, dtype=torch.int64, device=DEV)
    # norm: one rounding to 32 bits of a sum in 64 (squares and sums: 1e-16 each, a few million of them at most)
    for dest in (out, None):
        got = clip(grads, max_norm, out=dest, status=status)
        assert abs(got[0] - norm) <= 1.01 * U32 * norm and abs(got[1] - factor) <= 1.01 * U32 * factor and int(status) == 0
        if dest is not None:
            assert all(torch.equal(g, k) for g, k in zip(grads, kept))
            want = np.concatenate(before) * factor
            assert np.all(np.abs(f64(out) - want) <= 2.1 * U32 * np.abs(want))
    for g, b, k in zip(grads, before, kept):
        if factor == 1.0:
            assert torch.equal(g, k)
        else:
            assert np.all(np.abs(f64(g) - b * factor) <= (2.1 * U32 + (U16 * 1.001 if g.dtype == torch.bfloat16 else 0)) * np.abs(b * factor))


def test_clipping_of_views_that_begin_anywhere():
    whole32, whole16 = values(1, 70000), values(2, 70000).to(torch.bfloat16)
    grads, marks = [], []
    for off, n in ((1, 20001), (20003, 9000), (30002, 8195)):
        for w in (whole32, whole16):
            grads.append(w[off:off + n]); marks.append((w, off, n))
    before = [f64(g) for g in grads]
    outside = [w.clone() for w in (whole32, whole16)]
    norm = np.sqrt(sum(float(np.sum(b * b)) for b in before))
    big = torch.full((sum(g.numel() for g in grads) + 3,), 4.0, device=DEV)
    clip(grads, 2.0, out=big[1:-2])
    want = np.concatenate(before) * (2.0 / (norm + 1e-6))
    assert np.all(np.abs(f64(big[1:-2]) - want) <= 2.1 * U32 * np.abs(want)) and float(big[0]) == 4.0 and bool((big[-2:] == 4.0).all())
    clip(grads, 2.0)
    for w, old in zip((whole32, whole16), outside):
        inside = torch.zeros(70000, dtype=torch.bool, device=DEV)
        for ww, off, n in marks:
            if ww is w:
                inside[off:off + n] = True
        assert torch.equal(w[~inside], old[~inside])
    for g, b in zip(grads, before):
        assert np.all(np.abs(f64(g) - b * (2.0 / (norm + 1e-6))) <= (2.1 * U32 + U16 * 1.001) * np.abs(b))


def test_clipping_of_unusual_values():
    huge = torch.full((5000,), 3e30, device=DEV)              # squares beyond 32 bits
    got = clip([huge], 1.0)
    assert abs(got[0] / (np.sqrt(5000.0) * 3e30) - 1) < 1e-6 and abs(got[1] * np.sqrt(5000.0) * 3e30 - 1) < 1e-6
    tiny = torch.full((5000,), 1e-30, device=DEV)
    assert abs(clip([tiny], 1e-31)[0] / (1e-30 * np.sqrt(5000.0)) - 1) < 1e-6
    zero = torch.zeros(100, device=DEV)
    assert tuple(clip([zero], 1.0)) == (0.0, 1.0)
    assert tuple(clip([], 1.0)) == (0.0, 1.0)
    for bad in (float("nan"), float("inf")):
        g = [values(1, 1000), values(2, 500).to(torch.bfloat16)]
        g[1][3] = bad
        kept = [t.clone() for t in g]
        status, out = torch.zeros(1, dtype=torch.int64, device=DEV), torch.empty(1500, device=DEV)
        for dest in (None, out):
            got = clip(g, 1.0, out=dest, status=status)
            assert not np.isfinite(got[0]) and got[1] == 1.0 and int(status) == 1
        assert all(torch.equal(a.float().nan_to_num(7.0), b.float().nan_to_num(7.0)) for a, b in zip(g, kept))
        assert torch.equal(out.nan_to_num(7.0), torch.cat([t.float() for t in kept]).nan_to_num(7.0))
    g = [values(3, 3000)]
    kept = g[0].clone()
    norm = clip(g, float("inf"))
    assert norm[1] == 1.0 and torch.equal(g[0], kept) and abs(norm[0] / np.linalg.norm(f64(kept)) - 1) < 1e-6


def test_clipping_gives_the_same_bits():
    grads = gradients([70001, 5, 2 ** 20], 3, ("fp32", "bf16"))
    a, b = torch.empty(70006 + 2 ** 20, device=DEV), torch.empty(70006 + 2 ** 20, device=DEV)
    assert tuple(clip(grads, 0.1, out=a)) == tuple(clip(grads, 0.1, out=b)) and torch.equal(a, b)


@pytest.mark.parametrize("dy_t,grad_t", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "fp32"), ("bf16", "bf16")])
@pytest.mark.parametrize("n,V,d", [(1024, 300, 256), (1025, 300, 256), (1024, 131072, 24), (1024, 131073, 24), (700, 257, 1024), (700, 257, 1032), (700, 257, 2048), (700, 257, 2056),
                                   (333, 255, 250), (333, 256, 260), (1, 131072, 40), (63, 200000, 40), (1023, 30522, 264)])
def test_token_gradient_of_few_tokens(n, V, d, dy_t, grad_t):
    """Both sides of where one launch takes over from two: tokens, ids, slices of the columns (16-byte pieces or not) and bytes of the gradient, with
    long runs, with padding and on top of what is there."""
    for kind in ("zipf", "same", "runs"):
        dy, ids = values(n + d, n, d).to(T[dy_t]), token_ids(kind, n, V, n + V)
        got = grad_of(dy, ids, V, grad_t, scale=1.25)
        check_grad(dy, ids, V, got, 1.25)
        assert torch.equal(got, grad_of(dy, ids, V, grad_t, scale=1.25))
    ids = token_ids("zipf", n, V, 9)
    ids[::3] = 2
    dy[ids == 2] = float("nan")
    check_grad(torch.nan_to_num(dy.float()), ids, V, grad_of(dy, ids, V, grad_t, scale=0.5, pad_id=2), 0.5, pad=2)


@pytest.mark.parametrize("n", [0, 1, 700, 1024, 1025])
@pytest.mark.parametrize("V,d", [(300, 256), (131072, 64), (200000, 40)])
def test_token_gradient_of_few_tokens_on_top(n, V, d):
    from paper_2310_05674_amd import binding as B
    dy, ids = values(n + 1, n, d), token_ids("zipf", n, V, 3)
    grad = values(6, V, d)
    before = f64(grad)
    ws = torch.full((B.embedding_grad_bytes(n, V, d),), 0xa5, dtype=torch.uint8, device=DEV)
    B.op_embedding_grad(dy, ids, grad, ws, scale=0.75, accumulate=True)
    check_grad(dy, ids, V, grad, 0.75, start=before)
    unseen = np.setdiff1d(np.arange(V), ids.cpu().numpy())
    assert np.array_equal(f64(grad)[unseen], before[unseen])
    B.op_embedding_grad(dy, ids, grad, ws, scale=0.75)
    check_grad(dy, ids, V, grad, 0.75)


def test_tensors_that_the_binding_refuses():
    """On the host, wrong types, strided rows of values: the binding says so before the library sees a pointer."""
    from paper_2310_05674_amd import binding as B
    new = lambda *s, dtype=torch.float32, device=DEV: torch.zeros(*s, dtype=dtype, device=device)
    table, ids, out, grad = new(10, 8), new(5, dtype=torch.int32), new(5, 8), new(10, 8)
    ws, clip = new(B.embedding_grad_bytes(5, 10, 8), dtype=torch.uint8), new(B.grad_clip_bytes(), dtype=torch.uint8)
    norm, status = new(2), new(1, dtype=torch.int64)
    for bad in (dict(table=new(10, 8, device="cpu")), dict(out=new(5, 8, device="cpu")), dict(ids=ids.cpu()), dict(ids=ids.long()), dict(ids=new(4, dtype=torch.int32)), dict(out=new(5, 7)),
                dict(table=new(10, 16)[:, ::2]), dict(out=new(8, 5).t())):
        a = dict(dict(table=table, ids=ids, out=out), **bad)
        with pytest.raises(ValueError):
            B.op_embedding(a["table"], a["ids"], a["out"])
    for bad in (dict(dy=out.cpu()), dict(grad=grad.cpu()), dict(ids=ids.cpu()), dict(ws=ws.cpu()), dict(grad=new(10, 7)), dict(dy=new(5, 16)[:, ::2]), dict(ws=new(2 * ws.numel(), dtype=torch.uint8)[::2])):
        a = dict(dict(dy=out, ids=ids, grad=grad, ws=ws), **bad)
        with pytest.raises(ValueError):
            B.op_embedding_grad(a["dy"], a["ids"], a["grad"], a["ws"])
    for bad in (dict(g=[grad.cpu()]), dict(g=[new(8, 10).t()]), dict(norm=norm.cpu()), dict(norm=norm.double()), dict(out=new(80, device="cpu")), dict(out=new(79)), dict(status=status.cpu()),
                dict(status=status.int()), dict(ws=clip.cpu())):
        a = dict(dict(g=[grad], norm=norm, out=None, status=None, ws=clip), **bad)
        with pytest.raises(ValueError):
            B.op_grad_clip(a["g"], 1.0, a["norm"], a["ws"], out=a["out"], status=a["status"])
    for half in (table.half(), ):
        with pytest.raises(B.SamaError):
            B.op_embedding(half, ids, out)


def test_one_row_of_any_stride():
    """A matrix of one row has no stride to speak of: torch calls it contiguous whatever it is a row of, and the operators take it."""
    from paper_2310_05674_amd import binding as B
    t, d, F, V = torch.bfloat16, 136, 72, 40

    def row(seed, width):
        whole = torch.zeros(2, width, dtype=t, device=DEV)
        whole[:1, :d].copy_(values(seed, 1, d))
        return whole[:1, :d]

    scratch = lambda n: torch.empty(n, dtype=torch.uint8, device=DEV)
    new = lambda *s: torch.empty(*s, dtype=t, device=DEV)
    w_in, w_out = (values(1, 2 * F, d) * 0.1).to(t), (values(2, d, F) * 0.1).to(t)
    for width in (d + 1, 2 ** 21 + 8):                        # odd, and beyond what the strides of several rows may be
        x, dy, y, dx = (row(k, width) for k in (3, 4, 5, 6))
        assert x.is_contiguous() and x.stride(0) == width
        out = []
        for a, b, c, e in ((x, dy, y, dx), (new(1, d).copy_(x), new(1, d).copy_(dy), new(1, d), new(1, d))):
            hidden, saved, dwi, dwo = new(1, F), scratch(B.glu_ffn_saved_bytes(1, F, t)), new(2 * F, d), new(d, F)
            B.op_glu_ffn(a, w_in, w_out, c, hidden, scratch(B.glu_ffn_bytes(1, d, F, t)), saved=saved)
            B.op_glu_ffn_grad(b, a, w_in, w_out, hidden, saved, e, dwi, dwo, scratch(B.glu_ffn_grad_bytes(1, d, F, t)))
            out.append([v.clone() for v in (c, e, hidden, dwi, dwo)])
        assert all(torch.equal(p, q) for p, q in zip(*out))
        table, ids = values(7, V, d).to(t), torch.full((1,), 17, dtype=torch.int32, device=DEV)
        B.op_embedding(table, ids, y, scale=2.0)
        assert torch.equal(y[0], (table[17].float() * 2.0).to(t))
        grad = new(V, d)
        B.op_embedding_grad(dy, ids, grad, scratch(B.embedding_grad_bytes(1, V, d)))
        assert torch.equal(grad[17], dy[0]) and not grad[:17].any() and not grad[18:].any()


@pytest.mark.parametrize("grad_t", ["fp32", "bf16"])
def test_clipping_by_a_factor_below_the_normal_numbers(grad_t):
    """A norm of 2e40, which is beyond fp32, takes a factor of 5e-41, which fp32 holds in seventeen bits: the results keep theirs.  Two products, each with one
    rounding, of a factor rounded once; bf16 in place rounds once more."""
    g = torch.full((5000,), 3e38, device=DEV).to(T[grad_t])
    g[::7] *= -0.5; g[1::7] = 1e-3; g[2::7] = 0.0
    b = f64(g)
    norm = np.sqrt(np.sum(b * b))
    out, status = torch.empty(5000, device=DEV), torch.full((1,), 7, dtype=torch.int64, device=DEV)
    for dest in (out, None):
        got = clip([g], 1.0, out=dest, status=status)
        # the norm is known in 64 bits: it is finite and it clips; as an fp32 value it is infinite
        assert got[0] == np.inf and abs(got[1] * norm - 1) < 1e-4 and int(status) == 0
    for t in (out, g):
        bar = 3.1 * U32 + (U16 * 1.001 if t.dtype == torch.bfloat16 else 0)
        assert np.all(np.abs(f64(t) - b / norm) <= bar * np.abs(b / norm) + 2.0 ** -133), float(np.max(np.abs(f64(t) * norm - b) / (np.abs(b) + 1e-30)))


@pytest.mark.parametrize("max_norm", [0.5, 1e9])
@pytest.mark.parametrize("types", [("fp32",), ("bf16",), ("bf16", "fp32"), ("fp32", "bf16", "bf16")])
def test_clipping_by_blocks_of_several_units(types, max_norm):
    """More units of 32 KB than there are blocks: a block walks a run of them, over parts of units, over the ends of tensors and from one type to the other.  More
    tensors than a launch takes, so that the runs begin anew; every one begins off 16 bytes, and after the first odd one so does its place in `out`."""
    sizes = [2 ** 25 + 8191, 3, 2 ** 25 - 5, 16385, 1, 2 ** 23 + 77] + [8191 + 4099 * (k % 7) for k in range(120)] + [2 ** 24 + 1, 0, 40000]
    grads, total = [], sum(sizes)
    gen = torch.Generator(device=DEV).manual_seed(5)
    for k, n in enumerate(sizes):
        whole = torch.randn(n + 8, device=DEV, generator=gen).mul_(10.0 ** -(k % 3)).to(T[types[k % len(types)]])
        grads.append(whole[k % 4:k % 4 + n])
    units = sum(-(-n // (16384 if g.dtype == torch.bfloat16 else 8192)) for n, g in zip(sizes[:100], grads))
    assert units > 4096
    # norm in 64 bits on the GPU, tensor by tensor
    norm = float(sum((g.double() ** 2).sum() for g in grads) ** 0.5)
    factor = min(1.0, max_norm / (norm + 1e-6))
    before = [g.clone() for g in grads]
    out = torch.full((total + 1,), 3.0, device=DEV)[1:]
    for dest in (out, None):
        got = clip(grads, max_norm, out=dest)
        assert abs(got[0] - norm) <= 1.01 * U32 * norm and abs(got[1] - factor) <= 1.01 * U32 * factor
        at = 0
        for g, b in zip(grads, before):
            if dest is not None:
                assert torch.equal(g, b)
                got_g, bar = out[at:at + g.numel()], 2.1 * U32
            else:
                got_g, bar = g, 2.1 * U32 + (U16 * 1.001 if g.dtype == torch.bfloat16 else 0)
            at += g.numel()
            if factor == 1.0:
                assert torch.equal(got_g.float(), b.float())
            want = b.double() * factor
            assert bool(((got_g.double() - want).abs() <= bar * want.abs()).all())


@pytest.mark.parametrize("table_t,out_t", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "fp32"), ("bf16", "bf16")])
@pytest.mark.parametrize("n,V,d", [(32769, 50, 256), (4099, 60, 1030), (4097, 33, 2048), (1100003, 9, 1), (70001, 700, 120), (1048577, 3, 1030), (1048579, 3, 4104)])
def test_lookup_of_many(n, V, d, table_t, out_t):
    """Sizes where a thread takes four pieces at a time, whole ones and value by value; with more than 2^20 blocks of one row, where a block goes on to more rows, and
    outputs of more than 2^32 values; ids beyond the table, and padding."""
    from paper_2310_05674_amd import binding as B
    vec = 8 if table_t == out_t == "bf16" else 4
    pieces = d // vec if d % vec == 0 else d
    assert n * pieces >= 2 ** 20
    table = values(n + d, V, d).to(T[table_t])
    ids = token_ids("outside", n, V, n)
    out = torch.full((n + 1, d), 9.0, dtype=T[out_t], device=DEV)
    B.op_embedding(table, ids, out[:n], scale=1.7, pad_id=2)
    scaled = (table.float() * torch.tensor(1.7, device=DEV)).to(T[out_t])
    for i0 in range(0, n, 2 ** 17):
        t = ids[i0:i0 + 2 ** 17]
        want = scaled[t.clamp(0, V - 1).long()]
        want[t == 2] = 0
        assert torch.equal(out[i0:min(i0 + 2 ** 17, n)], want)
    assert bool((out[n] == 9.0).all())


@pytest.mark.parametrize("dy_t,grad_t", [("bf16", "bf16"), ("fp32", "fp32")])
def test_token_gradient_beyond_32_bits(dy_t, grad_t):
    """More than 2^31 values of dy and of the gradient: ids from the whole table, and again on top of what is there."""
    from paper_2310_05674_amd import binding as B
    n, V, d = 2 ** 21 + 7, 2 ** 21 + 5, 1032
    gen = torch.Generator(device=DEV).manual_seed(3)
    ids = torch.randint(0, V, (n,), device=DEV, generator=gen, dtype=torch.int32)
    ids[::5] = V - 1 - ids[::5] % 3                       # two hundred thousand tokens each of the last three
    dy = torch.randint(-1, 2, (n, d), device=DEV, generator=gen, dtype=torch.int8).to(T[dy_t])   # every sum is an integer, and exact in fp32
    grad = torch.full((V, d), 7.0, dtype=T[grad_t], device=DEV)
    ws = torch.empty(B.embedding_grad_bytes(n, V, d), dtype=torch.uint8, device=DEV)
    for accumulate in (False, True):
        B.op_embedding_grad(dy, ids, grad, ws, scale=2.0, accumulate=accumulate)
        for c in range(0, d, 258):
            want = torch.zeros(V, 258, device=DEV).index_add_(0, ids, dy[:, c:c + 258].float()).mul_(2.0).to(T[grad_t])
            if accumulate:
                want = (want.float() + torch.zeros(V, 258, device=DEV).index_add_(0, ids, dy[:, c:c + 258].float()).mul_(2.0)).to(T[grad_t])
            assert torch.equal(grad[:, c:c + 258], want)


def test_token_gradient_of_more_tokens_than_a_list_numbers():
    """More than 2^23 tokens to a wave of the sort, which then looks through them again, and a run over half a million workgroups."""
    from paper_2310_05674_amd import binding as B
    n, V = 2 ** 27 + 700 * 450 + 3, 700
    i = torch.arange(n, device=DEV, dtype=torch.int32)
    half = n // 2 // V * V
    ids = torch.where(i < half, 5, i % V)
    dy = torch.randint(-1, 2, (n, 1), device=DEV, generator=torch.Generator(device=DEV).manual_seed(1), dtype=torch.int8).float()   # sums are integers below 2^24
    grad = torch.full((V, 1), 7.0, device=DEV)
    ws = torch.empty(B.embedding_grad_bytes(n, V, 1), dtype=torch.uint8, device=DEV)
    B.op_embedding_grad(dy, ids, grad, ws, scale=1.0)
    want = torch.zeros(V, dtype=torch.float64, device=DEV)
    rest = dy[half:, 0].double()
    whole = len(rest) // V * V
    want += rest[:whole].view(-1, V).sum(0)
    want[:len(rest) - whole] += rest[whole:]
    want[5] += dy[:half, 0].double().sum()
    assert torch.equal(grad[:, 0].double(), want)
