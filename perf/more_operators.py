"""What more operators of a token model's step are measured on: rotary positions of several axes, attention inside documents (causal, with a
prefix, capped, biased by distance, few new tokens over long caches) with its gradients, and distillation from a teacher's top logits.

Each case is one call (a training form: a forward and a backward call) on inputs that lie on the GPU.  run() computes it in its plain form,
elementary torch operations in 32 bits rounded once at the end, or, where `own` is set, through the library's entry points.

Heads of 64 as in the repository's encoder workloads (4, 12 and 16 of them) and of other usual widths, its vocabularies (8192, 30522, 50304), its batches of 32 x 128
tokens, and longer sequences than its encoders take."""
import math

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # queries and keys of one text of 128 tokens, the small encoder's heads: a call of a few microseconds, where its latency counts
        dict(name="rotary_text", op="rotary", T=128, H=8, D=64, R=64, axes=1, far=0, pairs="half", inverse=False, dtype="fp32"),
        # a video's tokens with positions in time, height and width, queries and keys together
        dict(name="rotary_video", op="rotary", T=16384, H=32, D=64, R=64, axes=3, far=0, pairs="half", inverse=False, dtype="bf16"),
        # the gradient of a head that is rotated in part, neighbours in pairs, an odd number of tokens far into a long text
        dict(name="rotary_grad_far", op="rotary", T=5003, H=20, D=96, R=48, axes=1, far=1000003, pairs="neighbours", inverse=True, dtype="fp32"),
        # a training step on 19 short texts of 37 tokens, the small encoder's heads in fp32
        dict(name="attend_small", op="attend", T=703, docs=19, mix=0, tail=0, Hq=4, Hk=4, D=64, causal=False, prefix=0.0, cap=0.0, slopes=False,
             dtype="fp32", train=True),
        # scoring the batch of 32 x 128 tokens in fp32, as the passes at theta +- eps v do: texts of unequal length, padding behind the last one
        dict(name="attend_score", op="attend", T=4096, docs=41, mix=1, tail=301, Hq=12, Hk=12, D=64, causal=True, prefix=0.0, cap=0.0, slopes=True,
             dtype="fp32", train=False),
        # training on packed documents of unequal length, an odd number of tokens, shared key heads
        dict(name="attend_documents", op="attend", T=8111, docs=23, mix=2, tail=88, Hq=16, Hk=4, D=64, causal=True, prefix=0.0, cap=0.0, slopes=False,
             dtype="bf16", train=True),
        # training with capped scores, a bias by distance and a question before each answer that all of its text sees
        dict(name="attend_prefix_capped", op="attend", T=4096, docs=4, mix=3, tail=0, Hq=12, Hk=12, D=64, causal=True, prefix=0.4, cap=30.0, slopes=True,
             dtype="bf16", train=True),
        # one long document: the most work listed
        dict(name="attend_long", op="attend", T=8192, docs=1, mix=4, tail=0, Hq=16, Hk=8, D=128, causal=True, prefix=0.0, cap=0.0, slopes=False,
             dtype="bf16", train=True),
        # three texts that are written token by token, each over its own cache
        dict(name="attend_tokens", op="tokens", n=3, keys=24001, mix=5, Hq=16, Hk=4, D=128, cap=0.0, slopes=False, dtype="bf16"),
        # the losses of a text of 37 tokens against eight logits of a teacher
        dict(name="distill_text", op="distill", T=37, V=8192, K=8, tau=2.0, empty=0.0, dtype="fp32", train=False),
        # a training step on the batch of 32 x 128 tokens, a quarter of them padding without a teacher
        dict(name="distill_batch", op="distill", T=4096, V=30522, K=32, tau=2.0, empty=0.25, dtype="bf16", train=True),
        # a long batch in fp32 with one logit each: the cross-entropy of labels
        dict(name="distill_labels", op="distill", T=4093, V=50304, K=1, tau=1.0, empty=0.05, dtype="fp32", train=True),
    ]


def _log_int(rng, lo, hi):
    """An integer whose logarithm is spread evenly over [lo, hi]."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _cost(c):
    w = work(c)
    return w["flops"] / (5e14 if c["dtype"] != "fp32" else 5e13) + w["bytes"] / 4e12


def draw(rng):
    """One more case: tokens from one up, documents, heads, widths, masks, vocabularies and types over the ranges of the listed ones."""
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["rotary", "attend", "attend", "attend", "attend", "tokens", "tokens", "distill", "distill"])
        c = {"op": op, "dtype": rng.choice(["bf16", "bf16", "fp32"])}
        if op == "rotary":
            c["T"], c["H"] = _log_int(rng, 1, 16384), _log_int(rng, 1, 48)
            c["D"] = rng.choice([32, 64, 80, 96, 128])
            c["R"] = c["D"] if rng.random() < 0.7 else c["D"] // 2
            c["axes"], c["far"] = rng.choice([1, 2, 3]), rng.choice([0, 0, 4096, 1000003])
            c["pairs"], c["inverse"] = rng.choice(["half", "neighbours"]), rng.random() < 0.5
        elif op == "distill":
            c["T"], c["V"] = _log_int(rng, 1, 4096), _log_int(rng, 1000, 50304)
            c["K"], c["tau"] = _log_int(rng, 1, 128), rng.choice([1.0, 2.0, 4.0])
            c["empty"], c["train"] = rng.choice([0.0, 0.0, 0.25]), rng.random() < 0.6
        else:
            c["Hk"] = _log_int(rng, 1, 16)
            c["Hq"] = c["Hk"] * rng.choice([1, 1, 2, 3, 4, 8])
            c["D"] = rng.choice([32, 64, 64, 80, 96, 128, 128])
            c["mix"] = rng.randrange(1000)
            c["cap"], c["slopes"] = rng.choice([0.0, 0.0, 30.0]), rng.random() < 0.3
            if op == "tokens":
                c["n"], c["keys"] = _log_int(rng, 1, 32), _log_int(rng, 1, 32768)
            else:
                c["T"] = _log_int(rng, 1, 8192)
                c["docs"] = _log_int(rng, 1, max(1, c["T"] // 16))
                c["tail"] = c["T"] // 10 if rng.random() < 0.3 else 0
                c["causal"] = rng.random() < 0.7
                c["prefix"] = rng.choice([0.0, 0.3]) if c["causal"] else 0.0
                c["train"] = rng.random() < 0.6
        if op in ("attend", "tokens") and float(c["Hq"]) * (c["T"] if op == "attend" else c["n"]) * _keys(c) > 1.1e9:
            continue   # the plain form holds a score for every pair of tokens, of other documents too
        if _cost(c) <= most:
            return c


# ------------------------------------------------------------------------------------------------------ layouts
def _shares(total, parts, mix):
    """`parts` unequal lengths of at least one, a fixed mixture, that add up to `total`."""
    w = np.random.RandomState(mix).lognormal(0.0, 0.7, parts)
    ends = np.maximum(np.arange(1, parts + 1), np.round(np.cumsum(w) / w.sum() * (total - parts)).astype(np.int64) + np.arange(1, parts + 1))
    ends[-1] = total
    return np.diff(np.concatenate([[0], ends]))


def _documents(c):
    """The first token of each document and the end of the last."""
    if c["op"] == "attend":
        return np.concatenate([[0], np.cumsum(_shares(c["T"] - c["tail"], c["docs"], c["mix"]))])
    return np.concatenate([[0], np.cumsum(_caches(c)[0])])


def _caches(c):
    """Of each text that goes on: the room it has in the cache, a multiple of 64 rows, and how many of them are filled."""
    filled = _shares(c["n"] * c["keys"], c["n"], c["mix"])
    return (filled + 64) // 64 * 64, filled


def _keys(c):
    return c["T"] if c["op"] == "attend" else int(_caches(c)[0].sum())


def _ranges(c):
    """The keys [begin, end) that each query sees."""
    if c["op"] == "tokens":
        first = _documents(c)[:-1]
        return first, first + _caches(c)[1]
    first = _documents(c)
    size = np.diff(first)
    t = np.arange(c["T"])
    doc = np.searchsorted(first, t, side="right") - 1
    inside = doc < c["docs"]
    doc = np.minimum(doc, c["docs"] - 1)
    begin, end = first[doc], first[doc + 1]
    if c["causal"]:
        end = np.maximum(t + 1, begin + _prefixes(c)[doc])
    return np.where(inside, begin, 0), np.where(inside, end, 0)


def _prefixes(c):
    return np.floor(c["prefix"] * np.diff(_documents(c))).astype(np.int64)


def _sections(c):
    """How many of the pairs turn by each axis."""
    pairs = c["R"] // 2
    rest = pairs * 3 // 8 if c["axes"] == 3 else pairs // 2
    return [pairs - (c["axes"] - 1) * rest] + (c["axes"] - 1) * [rest]


# ------------------------------------------------------------------------------------------------------ preparation
def prepare(case, seed):
    """Inputs, outputs and the workspace a program keeps, all on the GPU."""
    c = case
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    t = _TYPES[c["dtype"]]

    def normal(*shape, std=1.0, dtype=t):
        return torch.randn(*shape, device="cuda", generator=gen).mul_(std).to(dtype)

    def empty(*shape, dtype=t):
        return torch.empty(*shape, device="cuda", dtype=dtype)

    def ints(a):
        return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32).cuda()

    st = {"case": c}
    if c["op"] == "rotary":
        n = torch.arange(c["T"], device="cuda", dtype=torch.int32)
        # positions of text run on; of images they are a grid of 27 columns, of video one of 18 rows for each moment too
        axes = [n] if c["axes"] == 1 else [n // 27, n % 27] if c["axes"] == 2 else [n // 486, n // 27 % 18, n % 27]
        st["positions"] = torch.stack(axes) + c["far"]
        st["x"], st["out"] = normal(c["T"], c["H"], c["D"]), empty(c["T"], c["H"], c["D"])
    elif c["op"] == "distill":
        T, V, K = c["T"], c["V"], c["K"]
        st["logits"] = normal(T, V, std=2.0)
        # a teacher that agrees with its student on most of what they say
        teacher, ids = torch.topk(st["logits"].float() + normal(T, V, std=1.0, dtype=torch.float32), K, dim=1)
        listed_ids = torch.rand(T, 1, device="cuda", generator=gen) >= c["empty"]   # a token without a teacher has no entries
        st["ids"], st["teacher"] = torch.where(listed_ids, ids, -1).to(torch.int32), teacher.contiguous()
        st["loss"], st["saved"] = empty(T, dtype=torch.float32), empty(T, 2, dtype=torch.float32)
        if c["train"]:   # each token's loss is weighted, as the weight net does, in a mean
            st["dloss"] = torch.rand(T, device="cuda", generator=gen) / T
            st["dlogits"] = empty(T, V)
    else:
        Hq, Hk, D = c["Hq"], c["Hk"], c["D"]
        # slopes 2^-8 / H, 2^-16 / H, ... of the heads
        st["slopes"] = torch.exp2(-8.0 * torch.arange(1, Hq + 1, device="cuda", dtype=torch.float32) / Hq) if c["slopes"] else None
        if c["op"] == "tokens":
            Tq, Tk = c["n"], _keys(c)
            st["q"], st["k"], st["v"] = normal(Tq, Hq, D), normal(Tk, Hk, D), normal(Tk, Hk, D)
            begin, end = _ranges(c)
            st["spans"], st["at"] = ints(np.stack([begin, end], 1)), ints(end - 1)   # a new token is the last of its text
        else:
            Tq = Tk = c["T"]
            # queries, keys and values are parts of one product's rows
            qkv = normal(Tq, Hq + 2 * Hk, D)
            st["q"], st["k"], st["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
            st["at"] = torch.arange(Tq, device="cuda", dtype=torch.int32)
            st["offsets"], st["prefix"], st["spans"] = ints(_documents(c)), ints(_prefixes(c)), empty(Tq, 2, dtype=torch.int32)
        st["out"] = empty(Tq, Hq, D)
        if c.get("train"):
            st["dout"], st["lse"] = normal(Tq, Hq, D, std=1e-3), empty(Tq, Hq, dtype=torch.float32)
            dqkv = empty(Tq, Hq + 2 * Hk, D)
            st["dq"], st["dk"], st["dv"] = dqkv[:, :Hq], dqkv[:, Hq:Hq + Hk], dqkv[:, Hq + Hk:]
    if own and c["op"] in ("attend", "tokens"):   # the scratch memory a program allocates once for its sizes
        from paper_2310_05674_amd import binding as B
        size = B.attention_bytes(Tq, Tk, Hq, Hk, D, t)
        if c.get("train"):
            size = max(size, B.attention_grad_bytes(Tq, Tk, Hq, Hk, D, t))
        st["ws"] = empty(max(int(size), 1), dtype=torch.uint8)
    return st


# ------------------------------------------------------------------------------------------------------ the measured call
def _plain_rotary(st):
    c, R = st["case"], st["case"]["R"]
    x = st["x"].float()
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), torch.tensor(_sections(c), device="cuda"))
    # angles in 64 bits: those of far positions have no digits left in 32
    rate = torch.exp(torch.arange(R // 2, device="cuda", dtype=torch.float64) * (-2.0 * math.log(10000.0) / R))
    angle = (st["positions"].double()[axis].t() * rate)[:, None, :]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    if c["inverse"]:
        sin = -sin
    if c["pairs"] == "half":
        a, b = x[..., :R // 2], x[..., R // 2:R]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([turned, x[..., R:]], -1).to(_TYPES[c["dtype"]])


def _plain_spans(st):
    """The keys [begin, end) that each query of packed documents sees: none behind the last one."""
    c, first = st["case"], st["offsets"].long()
    t = torch.arange(c["T"], device="cuda")
    doc = torch.searchsorted(first, t, right=True) - 1
    inside = (doc >= 0) & (doc < c["docs"])
    doc = doc.clamp(0, c["docs"] - 1)
    begin, end = first[doc], first[doc + 1]
    if c["causal"]:
        end = torch.minimum(end, torch.maximum(t + 1, begin + st["prefix"].long()[doc]))
    return (torch.stack([begin, end], 1) * inside[:, None]).to(torch.int32)


def _plain_attention(st):
    c, t = st["case"], _TYPES[st["case"]["dtype"]]
    Hq, Hk, D = c["Hq"], c["Hk"], c["D"]
    G, Tq, Tk = Hq // Hk, st["q"].shape[0], st["k"].shape[0]

    def grouped(x):   # [tokens, Hq, D] -> the rows of each key head, [Hk, G tokens, D]
        return x.float().permute(1, 0, 2).reshape(Hk, G * Tq, D)

    def by_token(x):
        return x.reshape(Hq, Tq, D).permute(1, 0, 2).to(t)

    q, k, v = grouped(st["q"]), st["k"].float().permute(1, 0, 2), st["v"].float().permute(1, 0, 2)
    key = torch.arange(Tk, device="cuda", dtype=torch.int32)
    spans = _plain_spans(st) if c["op"] == "attend" else st["spans"]
    s = torch.matmul(q, k.transpose(1, 2)).mul_(D ** -0.5)
    if c["cap"]:
        bent = torch.tanh(s / c["cap"])
        s = bent * c["cap"]
    s = s.view(Hk, G, Tq, Tk)
    if c["slopes"]:
        s -= st["slopes"].view(Hk, G, 1, 1) * (st["at"][:, None] - key).abs().float()
    s.masked_fill_((key < spans[:, :1]) | (key >= spans[:, 1:]), -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s.sub_(top.masked_fill_(top == -math.inf, 0.0)))
    p /= p.sum(-1, keepdim=True).clamp_(min=1e-30)     # a query that sees nothing gets nothing
    p = p.view(Hk, G * Tq, Tk)
    out = {"out": by_token(torch.matmul(p, v))}
    if c["op"] == "attend":
        out["spans"] = spans
    if not c.get("train"):
        return out
    do = grouped(st["dout"])
    dp = torch.matmul(do, v.transpose(1, 2))
    dp -= (p * dp).sum(-1, keepdim=True)
    dp *= p
    if c["cap"]:
        dp *= 1.0 - bent * bent
    dp *= D ** -0.5
    out["dq"] = by_token(torch.matmul(dp, k))
    out["dk"] = torch.matmul(dp.transpose(1, 2), q).permute(1, 0, 2).to(t)
    out["dv"] = torch.matmul(p.transpose(1, 2), do).permute(1, 0, 2).to(t)
    return out


def _plain_distill(st):
    c, tau = st["case"], st["case"]["tau"]
    there = st["ids"] >= 0
    some = there.any(1)
    z = st["logits"].float() / tau
    zmax = z.amax(1, keepdim=True)
    e = torch.exp(z - zmax)
    total = e.sum(1, keepdim=True)
    t = (st["teacher"] / tau).masked_fill(~there, -math.inf)
    tmax = t.amax(1, keepdim=True).masked_fill(~some[:, None], 0.0)
    te = torch.exp(t - tmax)
    tsum = te.sum(1, keepdim=True).clamp(min=1e-30)
    p = te / tsum
    ids = st["ids"].clamp(min=0).long()
    logq = z.gather(1, ids) - zmax - total.log()
    logp = (t - tmax - tsum.log()).masked_fill(~there, 0.0)
    out = {"loss": (p * (logp - logq)).sum(1) * (tau * tau)}
    if c["train"]:
        d = (e / total).mul_(some[:, None]).scatter_add_(1, ids, -p)
        out["dlogits"] = d.mul_((st["dloss"] * tau)[:, None]).to(_TYPES[c["dtype"]])
    return out


def run(state):
    st, c = state, state["case"]
    if not own:
        return _plain_rotary(st) if c["op"] == "rotary" else _plain_distill(st) if c["op"] == "distill" else _plain_attention(st)
    from paper_2310_05674_amd import binding as B
    if c["op"] == "rotary":
        B.op_rotary(st["x"], st["positions"], st["out"], sections=_sections(c), base=10000.0, neighbours=c["pairs"] == "neighbours", inverse=c["inverse"])
        return st["out"]
    if c["op"] == "distill":
        B.op_distill(st["logits"], st["ids"], st["teacher"], st["loss"], st["saved"], temperature=c["tau"])
        if not c["train"]:
            return {"loss": st["loss"]}
        B.op_distill_grad(st["logits"], st["ids"], st["teacher"], st["dloss"], st["saved"], st["dlogits"], temperature=c["tau"])
        return {"loss": st["loss"], "dlogits": st["dlogits"]}
    if c["op"] == "attend":   # the first layer of a batch: where its documents begin and end, for each query
        B.op_attention_spans(st["offsets"], st["spans"], causal=c["causal"], prefix=st["prefix"])
    B.op_attention(st["q"], st["k"], st["v"], st["out"], st["spans"], st["ws"], scale=c["D"] ** -0.5, cap=c["cap"], slopes=st["slopes"], at=st["at"],
                   lse=st.get("lse"))
    out = {"out": st["out"], "spans": st["spans"]} if c["op"] == "attend" else {"out": st["out"]}
    if not c.get("train"):
        return out
    B.op_attention_grad(st["dout"], st["q"], st["k"], st["v"], st["out"], st["lse"], st["spans"], st["dq"], st["dk"], st["dv"], st["ws"],
                        scale=c["D"] ** -0.5, cap=c["cap"], slopes=st["slopes"], at=st["at"])
    return {**out, "dq": st["dq"], "dk": st["dk"], "dv": st["dv"]}


# ------------------------------------------------------------------------------------------------------ what a pass needs
def work(case):
    """Bytes: inputs once and outputs once; operations: 4 D for each head and pair of a query and a key that it sees, 10 D more for the gradients (each of
    the seven products once), of the others a few for each value."""
    c = case
    size = 2.0 if c["dtype"] == "bf16" else 4.0
    if c["op"] == "rotary":
        values = float(c["T"]) * c["H"] * c["D"]
        return {"bytes": 2.0 * values * size + 4.0 * c["axes"] * c["T"], "flops": 3.0 * values}
    if c["op"] == "distill":
        values = float(c["T"]) * c["V"]
        return {"bytes": values * size * (2 if c["train"] else 1) + 8.0 * c["T"] * c["K"] + 8.0 * c["T"], "flops": values * (5.0 if c["train"] else 3.0)}
    begin, end = _ranges(c)
    seen = float(np.maximum(end - begin, 0).sum())
    queries = float(len(begin)) * c["Hq"] * c["D"]
    keys = float(_caches(c)[1].sum() if c["op"] == "tokens" else c["T"]) * c["Hk"] * c["D"]
    if not c.get("train"):
        return {"bytes": (2.0 * queries + 2.0 * keys) * size + 8.0 * len(begin), "flops": 4.0 * c["D"] * c["Hq"] * seen}
    return {"bytes": (4.0 * queries + 4.0 * keys) * size + 8.0 * len(begin), "flops": 14.0 * c["D"] * c["Hq"] * seen}


# ------------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    """The same outputs from the definitions, in 64 bits: a rotation as a product of complex numbers; attention for one text and head after the other, its gradients by
    automatic differentiation; distillation as the divergence of two distributions over the whole vocabulary, differentiated the same way."""
    c, st = case, prepare(case, seed)
    f64 = torch.float64
    if c["op"] == "rotary":
        R, out = c["R"], st["x"].double()
        first = 0
        for a, count in enumerate(_sections(c)):
            for i in range(first, first + count):
                turn = st["positions"][a].double() * 10000.0 ** (-2.0 * i / R)
                w = torch.polar(torch.ones_like(turn), -turn if c["inverse"] else turn)[:, None]
                x, y = (i, i + R // 2) if c["pairs"] == "half" else (2 * i, 2 * i + 1)
                z = torch.complex(out[:, :, x].clone(), out[:, :, y].clone()) * w
                out[:, :, x], out[:, :, y] = z.real, z.imag
            first += count
        return out
    if c["op"] == "distill":
        loss = torch.zeros(c["T"], device="cuda", dtype=f64)
        grad = torch.zeros(c["T"], c["V"], device="cuda", dtype=f64) if c["train"] else None
        rows = torch.nonzero(st["ids"][:, 0] >= 0).reshape(-1)
        for part in torch.split(rows, 512):
            z = st["logits"][part].double().requires_grad_()
            p = torch.softmax(st["teacher"][part].double() / c["tau"], 1)
            ids = st["ids"][part].long()
            logq = torch.log_softmax(z / c["tau"], 1)
            each = c["tau"] ** 2 * torch.sum(torch.xlogy(p, p) - p * logq.gather(1, ids), 1)
            loss[part] = each.detach()
            if c["train"]:
                grad[part] = torch.autograd.grad(each, z, st["dloss"][part].double())[0]
        return {"loss": loss, "dlogits": grad} if c["train"] else {"loss": loss}
    Hq, Hk, D = c["Hq"], c["Hk"], c["D"]
    train = bool(c.get("train"))
    begin, end = _ranges(c)
    names = ["out", "dq", "dk", "dv"] if train else ["out"]
    got = {n: torch.zeros(st[n].shape, device="cuda", dtype=f64) for n in names}
    if c["op"] == "attend":
        got["spans"] = torch.as_tensor(np.stack([begin, end], 1), dtype=torch.int32).cuda()
    first = _documents(c)
    for d in range(len(first) - 1):
        lo, hi = int(first[d]), int(first[d + 1])
        rows = slice(lo, hi) if c["op"] == "attend" else slice(d, d + 1)
        b, e = (torch.as_tensor(np.asarray(x[rows]), device="cuda")[:, None] for x in (begin, end))
        j = torch.arange(lo, hi, device="cuda")[None]
        hidden = torch.logical_or(j < b, j >= e)
        away = (st["at"][rows].long()[:, None] - j).abs().double()
        for h in range(Hq):
            q = st["q"][rows, h].double().requires_grad_(train)
            k = st["k"][lo:hi, h * Hk // Hq].double().requires_grad_(train)
            v = st["v"][lo:hi, h * Hk // Hq].double().requires_grad_(train)
            s = torch.mm(q, k.t()) / math.sqrt(D)
            if c["cap"]:
                s = c["cap"] * torch.tanh(s / c["cap"])
            if c["slopes"]:
                s = s - float(st["slopes"][h]) * away
            o = torch.mm(torch.softmax(s.masked_fill(hidden, -math.inf), 1), v)
            got["out"][rows, h] = o.detach()
            if train:
                dq, dk, dv = torch.autograd.grad(o, (q, k, v), st["dout"][rows, h].double())
                got["dq"][rows, h] = dq
                got["dk"][lo:hi, h * Hk // Hq] += dk
                got["dv"][lo:hi, h * Hk // Hq] += dv
    return got
