"""What the operators of a token model's base step are measured on: the embedding lookup with scaling and its gradient by sorted
tokens, the gated feed-forward block with its backward pass, and the global gradient norm with clipping.

Each case is one call (the training form of the feed-forward block: a forward and a backward call) on inputs that lie on the GPU.
run() computes it in its plain form, elementary torch operations in 32 bits rounded once at the end, or, where `own` is set, through
the library's entry points.

Widths, vocabularies, sequence lengths and batches are those of the repository's encoder workloads (4 x 256 with 8192 tokens, 12 x 768
with 30522, 24 x 1024 with 50265 and 50304) and ragged relatives of them; a gated block has three matrices for two, so that F is at
two thirds of the plain block's or as wide as it."""
import math

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # one text of 128 tokens through the small encoder's table: a call of a few microseconds, where its latency counts
        dict(name="lookup_text", op="lookup", n=128, V=8192, d=256, scale=16.0, pad=0.0, table="fp32", out="fp32"),
        # the activations of a batch of 32 texts of 1024 tokens, bf16 from the fp32 master table, a quarter padding
        dict(name="lookup_batch", op="lookup", n=32768, V=50265, d=1024, scale=32.0, pad=0.25, table="fp32", out="bf16"),
        # 19 short texts of 37 tokens: an odd number of rows, and a table whose zeros are most of the work
        dict(name="token_grad_small", op="token_grad", n=703, V=8192, d=256, scale=16.0, pad=0.0, dy="fp32", grad="fp32"),
        # the batch of 32 x 128 tokens that the 12 x 768 encoder trains on
        dict(name="token_grad_batch", op="token_grad", n=4096, V=30522, d=768, scale=1.0, pad=0.0, dy="fp32", grad="fp32"),
        # long sequences, bf16 activations' gradients, a quarter of them padding, an odd count
        dict(name="token_grad_long", op="token_grad", n=65521, V=50304, d=1024, scale=32.0, pad=0.25, dy="bf16", grad="fp32"),
        # one token at a time, as in serving: reading the weights is all there is to do
        dict(name="ffn_token", op="ffn", T=1, d=1024, F=4096, act="silu", dtype="bf16", train=False),
        # scoring a batch of 32 x 128 tokens
        dict(name="ffn_score", op="ffn", T=4096, d=768, F=2048, act="gelu", dtype="bf16", train=False),
        # a training step on an odd number of real tokens of padded texts, widths off the tiles
        dict(name="ffn_train_ragged", op="ffn", T=1021, d=520, F=1368, act="silu", dtype="bf16", train=True),
        # the largest batch of tokens the framework's encoders take, at the large model's widths: the most work listed
        dict(name="ffn_train_large", op="ffn", T=8192, d=1024, F=4096, act="silu", dtype="bf16", train=True),
        # the same operator in fp32, which the framework's MLPs train in
        dict(name="ffn_train_fp32", op="ffn", T=512, d=256, F=688, act="gelu", dtype="fp32", train=True),
        # clipping the small model's gradients: few bytes, a few dozen tensors
        dict(name="clip_small", op="clip", L=4, d=256, F=1024, V=8192, C=4, mixed=False, max_norm=1.0),
        # the 12 x 768 model's, matrices in bf16 and vectors in fp32, into the flat fp32 gradient the base solver takes
        dict(name="clip_large", op="clip", L=12, d=768, F=2048, V=30522, C=6, mixed=True, max_norm=1.0),
    ]


def _log_int(rng, lo, hi):
    """An integer whose logarithm is spread evenly over [lo, hi]."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _cost(c):
    w = work(c)
    return w["flops"] / (5e14 if c.get("dtype") != "fp32" else 5e13) + w["bytes"] / 4e12


def draw(rng):
    """One more case: numbers of tokens from one up, widths, vocabularies, depths and types over the ranges of the listed ones."""
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["lookup", "token_grad", "token_grad", "ffn", "ffn", "ffn", "clip"])
        c = {"op": op}
        if op in ("lookup", "token_grad"):
            c["n"] = _log_int(rng, 1, 65536)
            c["V"] = _log_int(rng, 1000, 50304)
            c["d"] = 8 * _log_int(rng, 8, 256) if rng.random() < 0.8 else _log_int(rng, 37, 1200)
            c["scale"] = rng.choice([1.0, round(math.sqrt(c["d"]), 3)])
            c["pad"] = rng.choice([0.0, 0.0, 0.25, 0.5])
            first, second = ("table", "out") if op == "lookup" else ("dy", "grad")
            c[first] = rng.choice(["bf16", "fp32"])
            c[second] = rng.choice(["bf16", "fp32"])
        elif op == "ffn":
            c["T"] = _log_int(rng, 1, 16384)
            c["d"] = 8 * _log_int(rng, 8, 256)
            c["F"] = 8 * max(8, int(c["d"] * (1.5 + 3 * rng.random()) / 8))
            c["act"] = rng.choice(["silu", "gelu"])
            c["dtype"] = rng.choice(["bf16", "bf16", "bf16", "fp32"])
            c["train"] = rng.random() < 0.6
        else:
            c["L"] = _log_int(rng, 1, 24)
            c["d"] = 8 * _log_int(rng, 8, 128)
            c["F"] = 8 * max(8, int(c["d"] * (1.5 + 3 * rng.random()) / 8))
            c["V"] = _log_int(rng, 1000, 50304)
            c["C"] = rng.randint(2, 9)
            c["mixed"] = rng.random() < 0.5
            c["max_norm"] = rng.choice([0.5, 1.0, 1e9])
        if _cost(c) <= most and 3072 not in c.values():
            return c


# ------------------------------------------------------------------------------------------------------ preparation
def _zipf(V):
    return np.arange(1, V, dtype=np.float64) ** -1.1


def _tokens(c, gen):
    """Ids as texts have them: Zipf(1.1) over 1..V-1; id 0 is the padding, the last positions."""
    cdf = torch.arange(1, c["V"], device="cuda", dtype=torch.float64).pow(-1.1).cumsum(0)
    u = torch.rand(c["n"], device="cuda", dtype=torch.float64, generator=gen) * cdf[-1]
    ids = (torch.searchsorted(cdf, u) + 1).clamp_(max=c["V"] - 1).to(torch.int32)
    real = c["n"] - int(c["pad"] * c["n"])
    ids[real:] = 0
    return ids


def _shapes(c):
    """The gradients of a token model: table, each layer's matrices and gains, the classifier."""
    d, F = c["d"], c["F"]
    layer = [(3 * d, d), (d, d), (2 * F, d), (d, F), (3 * d,), (d,), (d,), (d,)]
    return [(c["V"], d)] + c["L"] * layer + [(d,), (c["C"], d), (c["C"],)]


def prepare(case, seed):
    """Inputs, outputs and the workspace a program keeps, all on the GPU."""
    c = case
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.randn(*shape, device="cuda", generator=gen).mul_(std).to(dtype)

    def empty(*shape, dtype):
        return torch.empty(*shape, device="cuda", dtype=dtype)

    st = {"case": c}
    if c["op"] == "lookup":
        st["ids"] = _tokens(c, gen)
        st["table"] = normal(c["V"], c["d"], std=0.02, dtype=_TYPES[c["table"]])
        st["out"] = empty(c["n"], c["d"], dtype=_TYPES[c["out"]])
    elif c["op"] == "token_grad":
        st["ids"] = _tokens(c, gen)
        st["dy"] = normal(c["n"], c["d"], std=1e-3, dtype=_TYPES[c["dy"]])
        st["grad"] = empty(c["V"], c["d"], dtype=_TYPES[c["grad"]])
    elif c["op"] == "ffn":
        T, d, F, t = c["T"], c["d"], c["F"], _TYPES[c["dtype"]]
        st["x"] = normal(T, d, dtype=t)
        st["w_in"] = normal(2 * F, d, std=d ** -0.5, dtype=t)
        st["w_out"] = normal(d, F, std=F ** -0.5, dtype=t)
        st["y"], st["hidden"] = empty(T, d, dtype=t), empty(T, F, dtype=t)
        if c["train"]:
            st["dy"] = normal(T, d, std=1e-3, dtype=t)
            st["dx"], st["dw_in"], st["dw_out"] = empty(T, d, dtype=t), empty(2 * F, d, dtype=t), empty(d, F, dtype=t)
    else:
        big = torch.bfloat16 if c["mixed"] else torch.float32
        st["grads"] = [normal(*s, std=10.0 ** -(1 + k % 4), dtype=big if len(s) == 2 else torch.float32) for k, s in enumerate(_shapes(c))]
        st["out"] = empty(sum(g.numel() for g in st["grads"]), dtype=torch.float32)
        st["norm"] = empty(2, dtype=torch.float32)
    if own:   # the scratch memory a program allocates once for its sizes
        from paper_2310_05674_amd import binding as B

        def scratch(size):
            return empty(max(int(size), 1), dtype=torch.uint8)

        if c["op"] == "token_grad":
            st["ws"] = scratch(B.embedding_grad_bytes(c["n"], c["V"], c["d"]))
        elif c["op"] == "ffn":
            st["ws"] = scratch(B.glu_ffn_bytes(c["T"], c["d"], c["F"], _TYPES[c["dtype"]]))
            if c["train"]:
                st["saved"] = scratch(B.glu_ffn_saved_bytes(c["T"], c["F"], _TYPES[c["dtype"]]))
                st["ws_grad"] = scratch(B.glu_ffn_grad_bytes(c["T"], c["d"], c["F"], _TYPES[c["dtype"]]))
        elif c["op"] == "clip":
            st["ws"] = scratch(B.grad_clip_bytes())
    return st


# ------------------------------------------------------------------------------------------------------ the measured call
def _gate(act, g):
    """The activation of the gate and its derivative."""
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1.0 + g * (1.0 - s))
    phi = 0.5 * (1.0 + torch.erf(g * (1.0 / math.sqrt(2.0))))
    return g * phi, phi + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain(st):
    c = st["case"]
    if c["op"] == "lookup":
        rows = st["table"][st["ids"].clamp(0, c["V"] - 1).long()].float() * c["scale"]
        return rows.masked_fill_((st["ids"] == 0)[:, None], 0.0).to(_TYPES[c["out"]])
    if c["op"] == "token_grad":
        rows = (st["dy"].float() * c["scale"]).masked_fill_((st["ids"] == 0)[:, None], 0.0)
        grad = torch.zeros(c["V"], c["d"], device="cuda")
        grad.index_add_(0, st["ids"].clamp(0, c["V"] - 1), rows)
        return grad.to(_TYPES[c["grad"]])
    if c["op"] == "ffn":
        t, F = _TYPES[c["dtype"]], c["F"]
        x, w_in, w_out = st["x"].float(), st["w_in"].float(), st["w_out"].float()
        pre = x @ w_in.t()
        g, u = pre[:, :F], pre[:, F:]
        a, da = _gate(c["act"], g)
        h = a * u
        y = (h @ w_out.t()).to(t)
        if not c["train"]:
            return {"y": y}
        dy = st["dy"].float()
        dh = dy @ w_out
        dpre = torch.cat([dh * u * da, dh * a], 1)
        return {"y": y, "dx": (dpre @ w_in).to(t), "dw_in": (dpre.t() @ x).to(t), "dw_out": (dy.t() @ h).to(t)}
    flat = torch.cat([g.reshape(-1).float() for g in st["grads"]])
    norm = flat.square().sum().sqrt()
    factor = (c["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
    return {"norm": norm.reshape(1), "grad": flat * factor}


def run(state):
    if not own:
        return _plain(state)
    from paper_2310_05674_amd import binding as B
    st, c = state, state["case"]
    if c["op"] == "lookup":
        B.op_embedding(st["table"], st["ids"], st["out"], scale=c["scale"], pad_id=0)
        return st["out"]
    if c["op"] == "token_grad":
        B.op_embedding_grad(st["dy"], st["ids"], st["grad"], st["ws"], scale=c["scale"], pad_id=0)
        return st["grad"]
    if c["op"] == "ffn":
        if not c["train"]:
            B.op_glu_ffn(st["x"], st["w_in"], st["w_out"], st["y"], st["hidden"], st["ws"], act=c["act"])
            return {"y": st["y"]}
        B.op_glu_ffn(st["x"], st["w_in"], st["w_out"], st["y"], st["hidden"], st["ws"], act=c["act"], saved=st["saved"])
        B.op_glu_ffn_grad(st["dy"], st["x"], st["w_in"], st["w_out"], st["hidden"], st["saved"], st["dx"], st["dw_in"], st["dw_out"],
                          st["ws_grad"], act=c["act"])
        return {"y": st["y"], "dx": st["dx"], "dw_in": st["dw_in"], "dw_out": st["dw_out"]}
    B.op_grad_clip(st["grads"], c["max_norm"], st["norm"], st["ws"], out=st["out"])
    return {"norm": st["norm"][:1], "grad": st["out"]}


# ------------------------------------------------------------------------------------------------------ what a pass needs
def work(case):
    """Bytes: inputs once and outputs once (of a table, the rows that such a batch has: expected distinct ids); operations: 2 for
    each product and sum of the matrix products, of the others one a value."""
    c = case
    size = {"bf16": 2, "fp32": 4}
    if c["op"] in ("lookup", "token_grad"):
        real = c["n"] - int(c["pad"] * c["n"])
        if c["op"] == "token_grad":   # rows of padding need not be read, every row of the table's gradient is written
            return {"bytes": 4.0 * c["n"] + float(real) * c["d"] * size[c["dy"]] + float(c["V"]) * c["d"] * size[c["grad"]], "flops": float(real) * c["d"]}
        p = _zipf(c["V"])
        distinct = float(np.sum(-np.expm1(real * np.log1p(-p / p.sum()))))
        return {"bytes": 4.0 * c["n"] + distinct * c["d"] * size[c["table"]] + float(c["n"]) * c["d"] * size[c["out"]], "flops": float(real) * c["d"]}
    if c["op"] == "ffn":
        T, d, F = c["T"], c["d"], c["F"]
        weights, rows = 3.0 * d * F, 2.0 * T * d      # in and out; the gradients' are as many again
        return {"bytes": (weights + rows) * (2 if c["train"] else 1) * size[c["dtype"]], "flops": 6.0 * T * d * F * (3 if c["train"] else 1)}
    matrices = sum(s[0] * s[1] for s in _shapes(c) if len(s) == 2)
    vectors = sum(s[0] for s in _shapes(c) if len(s) == 1)
    return {"bytes": matrices * (6.0 if c["mixed"] else 8.0) + vectors * 8.0, "flops": 3.0 * (matrices + vectors)}


# ------------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    """The same outputs from the formulas, in 64 bits: a lookup as one scaled row a token, its gradient as the sum over the tokens of each
    id (sorted, by differences of the running sum's two ends), the block through the gate's formula and, backward, the chain rule."""
    c, st = case, prepare(case, seed)
    f64 = torch.float64
    if c["op"] == "lookup":
        out = torch.zeros(c["n"], c["d"], device="cuda", dtype=f64)
        real = torch.nonzero(st["ids"] != 0).reshape(-1)
        out[real] = torch.index_select(st["table"], 0, st["ids"][real]).double() * float(c["scale"])
        return out
    if c["op"] == "token_grad":
        real = torch.nonzero(st["ids"] != 0).reshape(-1)
        order = real[torch.argsort(st["ids"][real].long(), stable=True)]
        out = torch.zeros(c["V"], c["d"], device="cuda", dtype=f64)
        if order.numel() == 0:
            return out
        ids, count = torch.unique_consecutive(st["ids"][order].long(), return_counts=True)
        ends = count.cumsum(0)
        for k0 in range(0, c["d"], 128):   # a few columns at a time: the running sum takes 8 bytes a value
            run_sum = torch.cumsum(st["dy"][:, k0:k0 + 128].double()[order], 0)
            upto = run_sum[ends - 1]
            out[ids, k0:k0 + 128] = (upto - torch.cat([torch.zeros_like(upto[:1]), upto[:-1]])) * float(c["scale"])
        return out
    if c["op"] == "ffn":
        F = c["F"]
        x, w_in, w_out = st["x"].double(), st["w_in"].double(), st["w_out"].double()
        g, u = torch.mm(x, w_in[:F].t()), torch.mm(x, w_in[F:].t())
        if c["act"] == "silu":
            e = 1.0 / (1.0 + torch.exp(-g))
            a, da = g * e, e + g * e * (1.0 - e)
        else:
            e = 0.5 * torch.erfc(-g / math.sqrt(2.0))
            a, da = g * e, e + g * torch.exp(-g * g / 2.0) / math.sqrt(2.0 * math.pi)
        y = torch.mm(a * u, w_out.t())
        if not c["train"]:
            return {"y": y}
        dy = st["dy"].double()
        dh = torch.mm(dy, w_out)
        dg, du = dh * da * u, dh * a
        return {"y": y, "dx": torch.mm(dg, w_in[:F]) + torch.mm(du, w_in[F:]),
                "dw_in": torch.cat([torch.mm(dg.t(), x), torch.mm(du.t(), x)]), "dw_out": torch.mm(dy.t(), a * u)}
    parts = [g.double().reshape(-1) for g in st["grads"]]
    norm = math.sqrt(math.fsum(float(torch.dot(p, p)) for p in parts))
    factor = min(1.0, float(c["max_norm"]) / (norm + 1e-6))
    return {"norm": torch.tensor([norm], dtype=f64), "grad": torch.cat([p * factor for p in parts])}
