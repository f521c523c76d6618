"""Data reweighting on a small gated token model, out of the library's operators: python examples/gated_token_model.py [iterations]

The base learner is what modern text encoders are made of besides attention: a scaled embedding, gated feed-forward blocks with residual
connections, a mean over the real tokens and a linear classifier.  Each iteration is the method's: a base step on the noisy batch (the loss of
each text weighted by the net w(l; lambda)) with clipped gradients and Adam, the meta gradient on the clean batch, its adaptation, two forward passes at
theta +- eps v, and Adam on lambda with the finite difference of the two weight gradients.

  lookup      op_embedding       fp32 master table -> bf16 activations, padding gives zeros
  blocks      op_glu_ffn         and op_glu_ffn_grad, bf16 with fp32 sums, weights' gradients in fp32; the passes at theta +- eps v in fp32
  table       op_embedding_grad  by sorted tokens
  clipping    op_grad_clip       all tensors into the flat gradient
  solver      op_adam            refreshes the bf16 working copy of the matrices
  adaptation  op_adapt_norm, op_nudge

The flat parameter vector is laid out as the library lays its own out: all matrices of the blocks, then everything else."""
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch

from paper_2310_05674_amd import binding as B

PAD = 0


class GatedTokenModel:
    """Parameters, workspaces and one forward / backward pass for batches of up to `rows` tokens."""

    def __init__(self, V, d, F, layers, classes, rows, seed=0, act="silu"):
        self.V, self.d, self.F, self.L, self.C, self.rows, self.act = V, d, F, layers, classes, rows, act
        gen = torch.Generator(device="cuda").manual_seed(seed)
        shapes = [((2 * F, d), d ** -0.5) if k % 2 == 0 else ((d, F), (2 * layers * F) ** -0.5) for k in range(2 * layers)]
        shapes += [((V, d), d ** -0.5), ((classes, d), d ** -0.5)]
        self.theta = torch.cat([(torch.randn(*s, device="cuda", generator=gen) * std).reshape(-1) for s, std in shapes])
        self.n, self.shapes = self.theta.numel(), [s for s, _ in shapes]
        self.n16 = layers * 3 * d * F                     # the blocks' matrices, which have a bf16 working copy
        self.theta16 = self.theta[:self.n16].to(torch.bfloat16)
        self.m, self.v, self.g, self.vdir = (torch.zeros(self.n, device="cuda") for _ in range(4))
        self.t = 0
        bf16, byte = torch.bfloat16, torch.uint8
        new = lambda *s, dtype: torch.empty(*s, device="cuda", dtype=dtype)
        self.hidden = [new(rows, F, dtype=bf16) for _ in range(layers)]
        self.saved = [new(B.glu_ffn_saved_bytes(rows, F, bf16), dtype=byte) for _ in range(layers)]
        self.x = [new(rows, d, dtype=bf16) for _ in range(layers + 1)]
        self.grads = [new(*s, dtype=torch.float32) for s in self.shapes]
        self.ws = new(max(B.glu_ffn_bytes(rows, d, F, bf16), B.glu_ffn_grad_bytes(rows, d, F, bf16), B.embedding_grad_bytes(rows, V, d), B.grad_clip_bytes()), dtype=byte)
        self.norm, self.status = new(2, dtype=torch.float32), torch.zeros(1, dtype=torch.int64, device="cuda")
        self.partial, self.eps = new(65536, dtype=torch.float64), torch.zeros(2, device="cuda")

    def views(self, flat):
        out, at = [], 0
        for s in self.shapes:
            n = s[0] * s[1]
            if at + n > flat.numel():
                break
            out.append(flat[at:at + n].view(s))
            at += n
        return out

    def share(self, ids):
        """What each token is of its text's mean."""
        real = (ids != PAD).float()
        return real / real.sum(1, keepdim=True)

    def forward(self, ids, keep=True):
        """logits [n, C] of ids [n, S]; `keep`: for a backward pass."""
        n, S = ids.shape
        T = n * S
        master, work = self.views(self.theta), self.views(self.theta16)
        B.op_embedding(master[2 * self.L], ids.view(-1), self.x[0][:T], scale=self.d ** 0.5, pad_id=PAD)
        for l in range(self.L):
            y = self.x[l + 1][:T]
            B.op_glu_ffn(self.x[l][:T], work[2 * l], work[2 * l + 1], y, self.hidden[l][:T], self.ws, act=self.act, saved=self.saved[l] if keep else None)
            y += self.x[l][:T]
        self.pooled = torch.bmm(self.share(ids)[:, None, :], self.x[self.L][:T].view(n, S, self.d).float())[:, 0]
        return self.pooled @ master[-1].t()

    def forward_at(self, ids, theta):
        """logits at other parameters, in fp32: theta +- eps v differs from theta by less than half a bf16 ulp of most weights."""
        n, S = ids.shape
        T = n * S
        p = self.views(theta)
        new = lambda *s: torch.empty(*s, device="cuda")
        x, y, hidden = new(T, self.d), new(T, self.d), new(T, self.F)
        ws = torch.empty(B.glu_ffn_bytes(T, self.d, self.F, torch.float32), dtype=torch.uint8, device="cuda")
        B.op_embedding(p[2 * self.L], ids.view(-1), x, scale=self.d ** 0.5, pad_id=PAD)
        for l in range(self.L):
            B.op_glu_ffn(x, p[2 * l], p[2 * l + 1], y, hidden, ws, act=self.act)
            x += y
        return torch.bmm(self.share(ids)[:, None, :], x.view(n, S, self.d))[:, 0] @ p[-1].t()

    def backward(self, ids, dlogits):
        """Gradients of sum(dlogits * logits) of the last forward pass into self.grads."""
        n, S = ids.shape
        T = n * S
        work, master = self.views(self.theta16), self.views(self.theta)
        torch.mm(dlogits.t(), self.pooled, out=self.grads[-1])
        dx = (self.share(ids)[:, :, None] * (dlogits @ master[-1])[:, None, :]).reshape(T, self.d).to(torch.bfloat16)
        for l in reversed(range(self.L)):
            dx_in = torch.empty_like(dx)
            B.op_glu_ffn_grad(dx, self.x[l][:T], work[2 * l], work[2 * l + 1], self.hidden[l][:T], self.saved[l], dx_in, self.grads[2 * l],
                              self.grads[2 * l + 1], self.ws, act=self.act)
            dx += dx_in
        B.op_embedding_grad(dx, ids.view(-1), self.grads[2 * self.L], self.ws, scale=self.d ** 0.5, pad_id=PAD)

    def step(self, lr, max_norm):
        """Clips self.grads to a global norm, into the flat gradient, and takes an Adam step with it."""
        B.op_grad_clip(self.grads, max_norm, self.norm, self.ws, out=self.g, status=self.status)
        self.t += 1
        B.op_adam(self.g, self.m, self.v, self.theta, self.theta16, self.n16, self.t, lr, 0.9, 0.999, 1e-8)

    def adapt(self, lr, alpha):
        """v = (du / dg) . g_meta for the meta gradient in self.grads, and eps = alpha / ||v|| (self.eps[0])."""
        gmeta = torch.cat([g.reshape(-1) for g in self.grads])
        B.op_adapt_norm(self.g, self.m, self.v, gmeta, self.vdir, self.partial, self.t, lr, 0.9, 0.999, 1e-8, alpha, self.eps, self.status)

    def nudge(self):
        B.op_nudge(self.theta, self.vdir, self.eps, self.theta16, self.n16)


class WeightNet:
    """w(l; lambda) = sigmoid(W2 relu(W1 l + b1) + b2), its gradient in lambda and Adam on it.

    It starts flat and moves slowly: the losses at theta +- eps v move the net's input as well as what it multiplies, so the finite difference is of
    w'(l) l + w, which has the sign of w only while the net is not steep where it is saturated."""

    def __init__(self, H, lr, seed=1):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        n = lambda k, std=1.0: torch.randn(k, device="cuda", generator=gen) * std
        self.p = [n(H, 0.3), n(H), n(H, 0.3 * H ** -0.5), torch.zeros(1, device="cuda")]
        self.m, self.s = [torch.zeros_like(p) for p in self.p], [torch.zeros_like(p) for p in self.p]
        self.lr, self.t = lr, 0

    def __call__(self, losses):
        self.h = torch.relu(losses[:, None] * self.p[0] + self.p[1])
        return torch.sigmoid(self.h @ self.p[2] + self.p[3])

    def grad(self, losses):
        """d/dlambda of mean(w(l) l)."""
        w = self(losses)
        dz = w * (1 - w) * losses / losses.numel()
        dh = (dz[:, None] * self.p[2]) * (self.h > 0)
        return [(dh * losses[:, None]).sum(0), dh.sum(0), self.h.t() @ dz, dz.sum()[None]]

    def step(self, grads):
        self.t += 1
        for p, m, s, g in zip(self.p, self.m, self.s, grads):
            m.mul_(0.9).add_(g, alpha=0.1)
            s.mul_(0.999).addcmul_(g, g, value=0.001)
            p.addcdiv_(m / (1 - 0.9 ** self.t), (s / (1 - 0.999 ** self.t)).sqrt_().add_(1e-8), value=-self.lr)


def cross_entropy(logits, y):
    """Loss of each sample, and its gradient in the logits."""
    logp = torch.log_softmax(logits, 1)
    rows = torch.arange(len(y), device=y.device)
    d = logp.exp()
    d[rows, y] -= 1.0
    return -logp[rows, y], d


def iteration(model, net, train, meta, lr=1e-3, alpha=0.1, max_norm=1.0):
    """One base step and one meta step; returns the mean training loss and the weights of the training texts."""
    (ids, y), (mids, my) = train, meta
    losses, d = cross_entropy(model.forward(ids), y)
    weights = net(losses)
    model.backward(ids, d * (weights / len(y))[:, None])
    model.step(lr, max_norm)
    _, d = cross_entropy(model.forward(mids), my)
    model.backward(mids, d / len(my))
    if model.t >= 2:                                   # after one step from zero moments the adaptation is nothing but rounding
        model.adapt(lr, alpha)
        plus, minus = (net.grad(cross_entropy(model.forward_at(ids, model.theta + s * model.eps[0] * model.vdir), y)[0]) for s in (1.0, -1.0))
        net.step([(b - a) / (2 * model.eps[0]) for a, b in zip(plus, minus)])
        model.nudge()
    return losses.mean(), weights


def texts(n, S, V, C, noise, seed, teacher):
    """Zipf tokens and padding; the class is the teacher's, of a share `noise` another one's."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    cdf = torch.arange(1, V, device="cuda", dtype=torch.float64).pow(-1.1).cumsum(0)
    ids = torch.searchsorted(cdf, torch.rand(n, S, device="cuda", dtype=torch.float64, generator=gen) * cdf[-1]).add_(1).clamp_(max=V - 1)
    length = torch.randint(S // 4, S + 1, (n, 1), device="cuda", generator=gen)
    ids[torch.arange(S, device="cuda")[None] >= length] = PAD
    clean = (teacher[ids] * (ids != PAD)[..., None]).sum(1).argmax(1)
    flip = torch.rand(n, device="cuda", generator=gen) < noise
    y = torch.where(flip, (clean + torch.randint(1, C, (n,), device="cuda", generator=gen)) % C, clean)
    return ids.to(torch.int32), y, flip


def main(iterations=60):
    V, S, C = 2000, 40, 4
    model, net = GatedTokenModel(V, 128, 344, 2, C, rows=64 * S), WeightNet(32, 3e-3)
    teacher = torch.randn(V, C, device="cuda", generator=torch.Generator(device="cuda").manual_seed(9))
    for it in range(iterations):
        ids, y, flip = texts(64, S, V, C, 0.3, 100 + it, teacher)
        mids, my, _ = texts(32, S, V, C, 0.0, 5000 + it, teacher)
        loss, w = iteration(model, net, (ids, y), (mids, my))
        if it % 10 == 0 or it == iterations - 1:
            print("iteration %3d  loss %.3f  gradient norm %.2f (factor %.2f)  mean weight of texts labelled right %.3f, wrong %.3f" % (
                it, float(loss), float(model.norm[0]), float(model.norm[1]), float(w[~flip].mean()), float(w[flip].mean())), flush=True)
    return model, net


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 60)
