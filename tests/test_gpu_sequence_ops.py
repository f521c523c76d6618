"""Rotary positions and distillation from a teacher's top logits, against plain implementations in 64 bits.

Tolerances.  u = 2^-24, r what rounding to the type costs at most (2^-8 in bf16, u in fp32).
Rotary: the angle is right to 2^-49 turns for positions below 2^31 (a 64-bit product of at most 2^29 turns, the rate within 2^-50), cosine and sine are within 3 u of the exact (an eighth of a turn is
rounded once, u pi / 4 of angle, and sincospi has 2 u), two products and a sum: 6 u (|x| + |y|), and the store r |result|.
Distillation: an exponential of (z - top) / tau is off by (4 + 2 |z - top| / tau) u of itself, sums of V terms in runs of V / 256 by at most (V / 256 + 16) u: e_q for the softmax; loss by tau^2 (e_q + 2^-40
size of the terms) and its rounding u |loss|; dz by |g| tau (e_q q + 4 u p) and r |dz|."""
import math
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def step(t):
    return 2.0 ** -8 if t == torch.bfloat16 else U


# ------------------------------------------------------------------------------------------------------ rotary
def rotated(x, positions, sections, base, neighbours, inverse):
    """The rotation in 64 bits, and the sum of the sizes of what each value is made of."""
    R = 2 * sum(sections)
    y, size = x.double().clone(), x.double().abs()
    i = 0
    for a, count in enumerate(sections):
        for _ in range(count):
            turns = (positions.view(len(sections), -1)[a].double() * (base ** (-2.0 * i / R) / (2 * math.pi)))
            phi = 2 * math.pi * (turns - torch.round(turns))
            c, s = torch.cos(phi)[:, None], torch.sin(phi)[:, None] * (-1 if inverse else 1)
            p, q = (2 * i, 2 * i + 1) if neighbours else (i, i + R // 2)
            u, v = x[..., p].double(), x[..., q].double()
            y[..., p], y[..., q] = u * c - v * s, u * s + v * c
            size[..., p] = size[..., q] = u.abs() + v.abs()
            i += 1
    return y, size


def check_rotary(x, positions, sections, out, base=10000.0, neighbours=False, inverse=False):
    from paper_2310_05674_amd import binding as B
    kept = x.clone()
    B.op_rotary(x, positions, out, sections=sections, base=base, neighbours=neighbours, inverse=inverse)
    want, size = rotated(kept, positions, sections, base, neighbours, inverse)
    R = 2 * sum(sections)
    d = (out.double() - want).abs()
    # 2^-17 turns in 2^-49 ... of an angle: with positions below 2^24 it is nothing, of the largest 2^-20
    far = float(positions.abs().max()) * 2.0 ** -50 if positions.numel() else 0.0
    assert bool((d <= (6 * U + far) * size + step(x.dtype) * want.abs() * (1 + 2.0 ** -10) + 1e-40).all()), float((d - step(x.dtype) * want.abs()).max())
    assert torch.equal(out[..., R:], kept[..., R:])


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("T,H,D,sections", [(1, 1, 2, (1,)), (5, 3, 64, (32,)), (130, 8, 64, (12, 10, 10)), (777, 4, 80, (20,)), (33, 5, 7, (2, 1)), (40, 2, 256, (128,)), (3000, 12, 128, (16, 24, 24)),
                                            (64, 2, 48, (0, 12, 12)), (9, 300, 32, (4, 4, 4, 4))])
def test_rotary(T, H, D, sections, inverse, neighbours, t):
    gen = torch.Generator(device=DEV).manual_seed(T + D)
    x = torch.randn(T, H, D, device=DEV, generator=gen).to(TYPES[t])
    positions = torch.randint(-5, 5000, (len(sections), T), device=DEV, generator=gen, dtype=torch.int32)
    check_rotary(x, positions, sections, torch.empty_like(x), neighbours=neighbours, inverse=inverse)


@pytest.mark.parametrize("t", ["bf16", "fp32"])
def test_rotary_far_positions(t):
    x = torch.randn(6, 2, 64, device=DEV).to(TYPES[t])
    positions = torch.tensor([0, 1, 1000003, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=DEV)
    for base in (10000.0, 1e6, 0.5):
        check_rotary(x, positions, (32,), torch.empty_like(x), base=base if base > 1 else 10000.0)


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("neighbours", [False, True])
def test_rotary_in_place_and_strided(neighbours, t):
    gen = torch.Generator(device=DEV).manual_seed(1)
    rows = torch.randn(50, 9, 72, device=DEV, generator=gen).to(TYPES[t])
    kept = rows.clone()
    positions = torch.arange(50, device=DEV, dtype=torch.int32)
    for view in (rows[:, :6, :64], rows[:, 2:3, 4:68], rows[:, 1:4, 1:65], rows.transpose(0, 1)[:, :9, :64]):
        pos = torch.arange(view.shape[0], device=DEV, dtype=torch.int32)
        rows.copy_(kept)
        out = torch.empty(view.shape, device=DEV, dtype=TYPES[t])
        check_rotary(view, pos, (32,), out, neighbours=neighbours)
        assert torch.equal(rows, kept)
        check_rotary(view, pos, (32,), view, neighbours=neighbours)      # in place: the same
        assert torch.equal(view, out)
        view.copy_(out)
        changed = rows.clone()
        changed.copy_(kept)
        rest = torch.ones_like(rows, dtype=torch.bool)
        (rest[:, :6, :64] if view.shape[1] == 6 else rest[:, 2:3, 4:68] if view.shape[1] == 1 else rest[:, 1:4, 1:65] if view.shape[1] == 3 else rest.transpose(0, 1)[:, :9, :64]).fill_(False)
        assert torch.equal(rows[rest], kept[rest])                         # nothing beside the heads


def test_rotary_keeps_products_and_its_inverse_is_its_gradient():
    """q_i . k_j depends on i - j alone, and <R x, y> = <x, R' y>."""
    from paper_2310_05674_amd import binding as B
    gen = torch.Generator(device=DEV).manual_seed(2)
    x, y = (torch.randn(40, 2, 64, device=DEV, generator=gen) for _ in range(2))
    pos = torch.arange(100, 140, device=DEV, dtype=torch.int32)
    a, b = torch.empty_like(x), torch.empty_like(x)
    B.op_rotary(x, pos, a)
    B.op_rotary(y, pos, b, inverse=True)
    left, right = (a.double() * y.double()).sum(), (x.double() * b.double()).sum()
    assert abs(float(left - right)) <= 40 * 2 * 64 * 12 * U * 8
    q, k = x[:1].expand(40, 2, 64).contiguous(), y[:1].expand(40, 2, 64).contiguous()
    B.op_rotary(q, pos, a)
    B.op_rotary(k, pos + 7, b)
    dots = (a.double() * b.double()).sum(-1)
    size = (a.double().abs() * b.double().abs()).sum(-1).max()
    assert float((dots - dots[:1]).abs().max()) <= 64 * U * float(size)


# ------------------------------------------------------------------------------------------------------ distillation
def distilled(z, ids, teacher, tau, g):
    """loss, dlogits and their bounds in 64 bits."""
    T, V = z.shape
    there = (ids >= 0) & (ids < V) & (teacher != -math.inf)
    some = there.any(1)
    x = torch.where(some[:, None], z.double(), torch.zeros((), device=DEV, dtype=torch.float64)) / tau
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    log_q = x - top - torch.log(e.sum(1, keepdim=True))   # in this order: 3.4e38 + log 300 is 3.4e38 in 64 bits too
    q = torch.exp(log_q)
    reach = torch.where(q > 1e-30, (top - x).clamp(max=100), torch.zeros_like(x)).amax(1, keepdim=True)
    e_q = (4 + 2 * reach + V / 256 + 16) * U
    t = torch.where(there, teacher.double() / tau, torch.full((), -math.inf, device=DEV, dtype=torch.float64))
    p = torch.where(some[:, None], torch.softmax(t, 1), torch.zeros((), device=DEV, dtype=torch.float64))
    logp = torch.where(p > 0, torch.log(p.clamp(min=1e-300)), torch.zeros((), device=DEV, dtype=torch.float64))
    at = ids.clamp(0, V - 1).long()
    logq = log_q.gather(1, at)
    part = torch.where(p > 0, p * (logp - logq), torch.zeros((), device=DEV, dtype=torch.float64))
    loss = tau ** 2 * part.sum(1)
    eloss = tau ** 2 * (e_q[:, 0] + 2.0 ** -40 * (p * (logp.abs() + logq.abs().clamp(max=1e6))).sum(1)) + U * loss.abs()
    listed = torch.zeros_like(x).scatter_add_(1, at, torch.where(there, p, torch.zeros((), device=DEV, dtype=torch.float64)))
    grad = torch.where(some[:, None], g.double()[:, None] * tau * (q - listed), torch.zeros((), device=DEV, dtype=torch.float64))
    egrad = g.double().abs()[:, None] * tau * (2 * e_q * q + 6 * U * (listed + q)) + step(z.dtype) * grad.abs()
    return loss, eloss, grad, egrad


def check_distill(z, ids, teacher, tau, g=None, in_place=False, out=None):
    from paper_2310_05674_amd import binding as B
    T, V = z.shape
    g = torch.rand(T, device=DEV) + 0.1 if g is None else g
    loss, saved = torch.full((T,), 7.0, device=DEV), torch.full((T, 2), 7.0, device=DEV)
    kept = z.clone()
    B.op_distill(z, ids, teacher, loss, saved, temperature=tau)
    out = z if in_place else torch.full_like(z, 7.0) if out is None else out
    B.op_distill_grad(z, ids, teacher, g, saved, out, temperature=tau)
    want, tol, grad, gtol = distilled(kept, ids, teacher, tau, g)
    finite = torch.isfinite(want)
    assert bool(((loss.double() - want).abs() <= tol + 1e-37)[finite].all()), float(((loss.double() - want).abs() - tol).max())
    d = (out.double() - grad).abs()
    assert bool((d <= gtol * (1 + 2.0 ** -10) + 1e-37).all()), float((d - gtol).max())
    return loss, out


def entries(T, V, K, seed, empty=0.3):
    r = np.random.RandomState(seed)
    ids = r.randint(0, V, (T, K))
    ids[r.rand(T, K) < empty] = -1
    return torch.as_tensor(ids.astype(np.int32), device=DEV), torch.as_tensor((r.randn(T, K) * 3).astype(np.float32), device=DEV)


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("tau", [1.0, 2.5])
@pytest.mark.parametrize("T,V,K", [(1, 1, 1), (3, 7, 4), (5, 1000, 256), (37, 8192, 8), (600, 1531, 33), (9, 50304, 64), (2, 30522, 1), (700, 130, 65)])
def test_distill(T, V, K, tau, t):
    gen = torch.Generator(device=DEV).manual_seed(V)
    z = (torch.randn(T, V, device=DEV, generator=gen) * 3).to(TYPES[t])
    ids, teacher = entries(T, V, K, T)      # small vocabularies list ids several times
    _, out = check_distill(z, ids, teacher, tau)
    _, same = check_distill(z, ids, teacher, tau, in_place=True, g=None)
    assert same is z


@pytest.mark.parametrize("t", ["bf16", "fp32"])
def test_distill_strides_and_alignment(t):
    for V, ld, first, ldo, firsto in ((101, 104, 0, 104, 0), (101, 101, 1, 101, 3), (512, 520, 8, 516, 4), (1030, 1031, 5, 1033, 6)):
        whole = torch.randn(first + 20 * ld, device=DEV).to(TYPES[t])
        z = whole[first:].view(20, ld)[:, :V]
        to = torch.full((firsto + 20 * ldo,), 7.0, device=DEV, dtype=TYPES[t])
        out = to[firsto:].view(20, ldo)[:, :V]
        ids, teacher = entries(20, V, 5, V)
        check_distill(z, ids, teacher, 1.5, out=out)
        rest = to.clone()
        rest[firsto:].view(20, ldo)[:, :V] = 7
        assert bool((rest == 7).all())


@pytest.mark.parametrize("t", ["bf16", "fp32"])
def test_distill_unusual_values(t):
    """Masked vocabularies (minus infinity, the lowest number), a row that is nothing but such, tokens without entries over logits that hold anything, entries of minus infinity or NaN that are none."""
    T, V, K = 12, 300, 6
    z = torch.randn(T, V, device=DEV).to(TYPES[t])
    ids, teacher = entries(T, V, K, 5, empty=0.0)
    z[0, 10:] = -math.inf; ids[0] = torch.arange(K, device=DEV)
    z[1, 10:] = torch.finfo(TYPES[t]).min; ids[1] = torch.arange(K, device=DEV)
    z[2] = torch.finfo(TYPES[t]).min
    z[3] = float("nan"); ids[3] = -1; teacher[3] = float("nan")
    z[4] = math.inf; ids[4] = V
    teacher[5, 1:] = -math.inf
    teacher[6, 2] = float("nan"); ids[6, 2] = -7
    teacher[7] = -math.inf; z[7] = float("nan")
    ids[8] = 17                                           # the same id K times
    z[9] = 1e4; z[9, 3] = 2e4
    loss, out = check_distill(z, ids, teacher, 2.0)
    assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(out).all())
    for i in (3, 4, 7):
        assert float(loss[i]) == 0.0 and bool((out[i] == 0).all())
    z[10, 7], ids[10, 0] = -math.inf, 7                   # the teacher lists what the student rules out
    loss, _ = check_distill(z, ids, teacher, 2.0)
    assert float(loss[10]) == math.inf
    z[11, 3] = float("nan")
    loss, saved = torch.empty(T, device=DEV), torch.empty(T, 2, device=DEV)
    from paper_2310_05674_amd import binding as B
    B.op_distill(z, ids, teacher, loss, saved, temperature=2.0)
    assert bool(torch.isnan(loss[11])) and bool(torch.isfinite(loss[:10]).all())


def test_distill_of_one_label_is_the_cross_entropy():
    z = torch.randn(64, 999, device=DEV)
    y = torch.randint(0, 999, (64,), device=DEV)
    loss, _ = check_distill(z, y[:, None].to(torch.int32), torch.zeros(64, 1, device=DEV), 1.0)
    want = torch.nn.functional.cross_entropy(z.double(), y, reduction="none")
    assert float((loss.double() - want).abs().max()) < (4 + 20 + 999 / 256 + 16) * U + 16 * U


def test_distill_gradient_against_differences():
    """Central differences of the loss itself, in 64 bits of the formula and with the library's own fp32 losses."""
    T, V, K, tau = 4, 50, 5, 2.0
    z = torch.randn(T, V, device=DEV)
    ids, teacher = entries(T, V, K, 8)
    g = torch.ones(T, device=DEV)
    _, out = check_distill(z, ids, teacher, tau, g=g)
    h = 2.0 ** -5
    for j in (0, 3, int(ids[0].max()), 49):
        lo, hi = z.clone(), z.clone()
        lo[:, j] -= h; hi[:, j] += h
        a, b = check_distill(lo, ids, teacher, tau, g=g)[0], check_distill(hi, ids, teacher, tau, g=g)[0]
        # third derivative at most 1 / tau, differences of losses of up to 40
        assert float(((b - a).double() / (2 * h) - out[:, j].double()).abs().max()) <= h * h / 6 + 40 * 60 * U / h


# ------------------------------------------------------------------------------------------------------ together
def chain(B, x, w, pos, spans, ids, teacher, wl, bufs):
    """A layer's positions and attention, the vocabulary's product, the loss and back to the product's rows."""
    qkv, out, lse, ws, logits, loss, saved, dloss, dx, dqkv = bufs
    H, D = 4, 64
    torch.mm(x, w, out=qkv.view(len(x), -1))
    B.op_rotary(qkv[:, :2 * H], pos, qkv[:, :2 * H], sections=(16, 8, 8))
    B.op_attention(qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:], out, spans, ws, lse=lse, cap=30.0)
    torch.mm(out.view(len(x), -1), wl, out=logits)
    B.op_distill(logits, ids, teacher, loss, saved, temperature=2.0)
    B.op_distill_grad(logits, ids, teacher, dloss, saved, logits, temperature=2.0)
    torch.mm(logits, wl.t(), out=dx.view(len(x), -1))
    B.op_attention_grad(dx, qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:], out, lse, spans, dqkv[:, :H], dqkv[:, H:2 * H], dqkv[:, 2 * H:], ws, cap=30.0)
    B.op_rotary(dqkv[:, :2 * H], pos, dqkv[:, :2 * H], sections=(16, 8, 8), inverse=True)


def chain_setup(T, V, K, t):
    from paper_2310_05674_amd import binding as B
    H, D = 4, 64
    gen = torch.Generator(device=DEV).manual_seed(T)
    new = lambda *s, dtype=t: torch.empty(*s, device=DEV, dtype=dtype)
    x, w = torch.randn(T, H * D, device=DEV, generator=gen).to(t), (torch.randn(H * D, 3 * H * D, device=DEV, generator=gen) / 16).to(t)
    wl = (torch.randn(H * D, V, device=DEV, generator=gen) / 4).to(t)
    pos = torch.stack([torch.arange(T, device=DEV) // 16, torch.arange(T, device=DEV) // 4 % 4, torch.arange(T, device=DEV) % 4]).to(torch.int32)
    offsets, spans = torch.tensor([0, T // 3, T - 5], dtype=torch.int32, device=DEV), new(T, 2, dtype=torch.int32)
    B.op_attention_spans(offsets, spans, causal=True)
    ids, teacher = entries(T, V, K, T)
    size = (T, T, H, H, D, t)
    ws = new(max(B.attention_bytes(*size), B.attention_grad_bytes(*size)), dtype=torch.uint8)
    f32 = torch.float32
    bufs = (new(T, 3 * H, D), new(T, H, D), new(T, H, dtype=f32), ws, new(T, V), new(T, dtype=f32), new(T, 2, dtype=f32), torch.rand(T, device=DEV, generator=gen), new(T, H, D), new(T, 3 * H, D))
    return B, x, w, pos, spans, ids, teacher, wl, bufs


def test_a_run_of_them_against_automatic_differentiation():
    """fp32.  Tolerance: every stage is off by at most some 100 u of the sizes it sums, four stages follow one another and amplify by at most 10 each here: 1e-4 of the largest value."""
    T, V, K, H, D = 123, 501, 7, 4, 64
    B, x, w, pos, spans, ids, teacher, wl, bufs = chain_setup(T, V, K, torch.float32)
    chain(B, x, w, pos, spans, ids, teacher, wl, bufs)
    qkv = (x.double() @ w.double()).requires_grad_()
    a = qkv.view(T, 3 * H, D)
    rate = 10000.0 ** (-torch.arange(32, device=DEV, dtype=torch.float64) / 32)
    phi = (pos.double()[torch.tensor([0] * 16 + [1] * 8 + [2] * 8, device=DEV)].t() * rate)[:, None]
    qk = a[:, :2 * H]
    turned = torch.cat([qk[..., :32] * phi.cos() - qk[..., 32:] * phi.sin(), qk[..., :32] * phi.sin() + qk[..., 32:] * phi.cos()], -1)
    q, k, v = (m.transpose(0, 1) for m in (turned[:, :H], turned[:, H:], a[:, 2 * H:]))
    j = torch.arange(T, device=DEV)
    see = (j[None] >= spans[:, :1]) & (j[None] < spans[:, 1:])
    s = 30 * torch.tanh(torch.bmm(q, k.transpose(1, 2).contiguous()) / 8 / 30)
    s = torch.where(see, s, torch.full((), -1e300, device=DEV, dtype=torch.float64))
    p = torch.softmax(s, -1) * see.any(1)[:, None]
    z = torch.bmm(p, v.contiguous()).transpose(0, 1).reshape(T, -1) @ wl.double()
    there = ids >= 0
    t = torch.softmax(torch.where(there, teacher.double() / 2, torch.full((), -1e300, device=DEV, dtype=torch.float64)), 1) * there
    loss = 4 * (torch.xlogy(t, t) - t * torch.log_softmax(z / 2, 1).gather(1, ids.clamp(min=0).long())).sum(1) * there.any(1)
    loss.backward(bufs[7].double())
    loss = loss.detach()
    assert float((bufs[5].double() - loss).abs().max()) < 1e-4 * float(loss.abs().max())
    assert float((bufs[9].view(T, -1).double() - qkv.grad).abs().max()) < 1e-4 * float(qkv.grad.abs().max())


@pytest.mark.parametrize("t", ["bf16", "fp32"])
def test_a_run_in_a_graph_and_on_another_stream(t):
    """Captured and replayed with other inputs between eager calls, each time the eager call's bits; two graphs with a workspace each."""
    runs = [chain_setup(T, 500, 6, TYPES[t]) for T in (130, 700)]
    want = []
    for r in runs:
        chain(*r)
        want.append([b.clone() for i, b in enumerate(r[-1]) if i != 3])
    side = torch.cuda.Stream()
    graphs = []
    for r in runs:
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            chain(*r)
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            chain(*r)
        graphs.append(g)
    for turn in range(4):
        for r, g, w in zip(runs, graphs, want):
            for i, b in enumerate(r[-1]):
                if i not in (3, 7):
                    b.zero_()
            r[1].mul_(2.0 if turn % 2 == 0 else 0.5)     # other inputs in between, and back
            g.replay()
            r[1].mul_(0.5 if turn % 2 == 0 else 2.0)
            g.replay()
            torch.cuda.synchronize()
            for b, x in zip([b for i, b in enumerate(r[-1]) if i != 3], w):
                assert torch.equal(b, x)
        chain(*runs[turn % 2])
    with torch.cuda.stream(side):
        for r in runs:
            chain(*r)
    side.synchronize()
    for r, w in zip(runs, want):
        for b, x in zip([b for i, b in enumerate(r[-1]) if i != 3], w):
            assert torch.equal(b, x)


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [2 ** 22 - 1, 2 ** 22])
def test_distill_of_the_most_tokens(T, t):
    """As many tokens as there may be: a workgroup each, more work items than one dimension of a launch holds."""
    V, K = 3, 2
    gen = torch.Generator(device=DEV).manual_seed(T)
    z = torch.randn(T, V, device=DEV, generator=gen).to(TYPES[t])
    ids = torch.randint(-1, V, (T, K), device=DEV, generator=gen, dtype=torch.int32)
    check_distill(z, ids, torch.randn(T, K, device=DEV, generator=gen), 1.5)


@pytest.mark.parametrize("t", ["bf16", "fp32"])
def test_distill_beyond_2_to_31_values(t):
    """The first row, the rows about value 2^31 and the last, of 33000 x 65537 logits in place, rows at every alignment."""
    from paper_2310_05674_amd import binding as B
    T, V, K = 33000, 65537, 5
    z = torch.empty(T, V, device=DEV, dtype=TYPES[t])
    gen = torch.Generator(device=DEV).manual_seed(9)
    for part in z.split(4096):
        part.copy_(torch.randn(part.shape, device=DEV, generator=gen))
    ids, teacher = entries(T, V, K, 3)
    at = torch.tensor([0, 2 ** 31 // V - 1, 2 ** 31 // V, 2 ** 31 // V + 1, T - 1], device=DEV)
    kept = z[at]
    g, loss, saved = torch.rand(T, device=DEV) + 0.1, torch.full((T,), 7.0, device=DEV), torch.full((T, 2), 7.0, device=DEV)
    B.op_distill(z, ids, teacher, loss, saved, temperature=2.0)
    B.op_distill_grad(z, ids, teacher, g, saved, z, temperature=2.0)
    want, tol, grad, gtol = distilled(kept, ids[at], teacher[at], 2.0, g[at])
    assert bool(((loss[at].double() - want).abs() <= tol).all())
    assert bool(((z[at].double() - grad).abs() <= gtol * (1 + 2.0 ** -10) + 1e-37).all())


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("neighbours", [False, True])
def test_rotary_beyond_2_to_31_values(neighbours, t):
    """33000 tokens of 512 heads of 128, in place and out of place: the first token, those about value 2^31 and the last."""
    from paper_2310_05674_amd import binding as B
    T, H, D = 33000, 512, 128
    x = torch.empty(T, H, D, device=DEV, dtype=TYPES[t])
    gen = torch.Generator(device=DEV).manual_seed(10)
    for part in x.split(4096):
        part.copy_(torch.randn(part.shape, device=DEV, generator=gen))
    positions = torch.arange(T, device=DEV, dtype=torch.int32)
    at = torch.tensor([0, 2 ** 15 - 1, 2 ** 15, 2 ** 15 + 1, T - 1], device=DEV)
    kept = x[at]
    out = torch.empty_like(x)
    B.op_rotary(x, positions, out, neighbours=neighbours)
    B.op_rotary(x, positions, x, neighbours=neighbours)
    want, size = rotated(kept, positions[at], (D // 2,), 10000.0, neighbours, False)
    for got in (out[at], x[at]):
        assert bool(((got.double() - want).abs() <= 6 * U * size + T * 2.0 ** -50 * size + step(x.dtype) * want.abs() * (1 + 2.0 ** -10) + 1e-40).all())


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("base,positions", [(0.5, [0, 1, 1000003, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31]), (1.0, [5, 2 ** 31 - 1, -2 ** 31]), (1e-6, [0, 1, -3, 999]), (1e300, [7, 2 ** 31 - 1])])
def test_rotary_bases(base, positions, t):
    """Bases whose rates grow with the pair, or vanish.  With v = 2^-53 the kernel's rate is off by (5 ln rate + 4) v of itself (a logarithm, its share of the pair, an exponential, 1 / 2 pi), the
    reference's by (ln rate + 4) v, and each product with the position by v: angles differ by (6 |ln rate| + 10) v of themselves, where turns have a fraction at all."""
    from paper_2310_05674_amd import binding as B
    D = 64
    x = torch.randn(len(positions), 2, D, device=DEV).to(TYPES[t])
    pos, out = torch.tensor(positions, dtype=torch.int32, device=DEV), torch.empty_like(x)
    for neighbours in (False, True):
        B.op_rotary(x, pos, out, base=base, neighbours=neighbours)
        want, size = rotated(x, pos, (D // 2,), base, neighbours, False)
        ln_rate = torch.arange(D // 2, device=DEV, dtype=torch.float64) * (-2.0 * math.log(base) / D)
        far = pos.double().abs()[:, None] * torch.exp(ln_rate) * (6 * ln_rate.abs() + 10) * 2.0 ** -53
        far = (far.repeat_interleave(2, 1) if neighbours else torch.cat([far, far], 1))[:, None]
        assert float(far.max()) < 2.0 ** -12                  # it says something
        assert bool(((out.double() - want).abs() <= (6 * U + far) * size + step(x.dtype) * want.abs() * (1 + 2.0 ** -10) + 1e-40).all())
