"""The example that runs the token model's operators together: its gradients against automatic differentiation in 64 bits, and that it learns."""
import importlib.util
import os
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("gated_token_model", os.path.join(ROOT, "examples", "gated_token_model.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("n,S,V,d,F,L,act", [(3, 7, 50, 64, 72, 1, "silu"), (9, 21, 300, 72, 136, 2, "gelu")])
def test_gradients(example, n, S, V, d, F, L, act):
    """Tolerance: activations and the gradients between blocks are rounded to bf16, about three times a block each way (stored sum, hidden, dg and
    du), 2^-8 at most and 1.66e-3 in the root mean square each; the blocks' weights in the graph are the rounded ones.  Nine of them for one block and eighteen for two, unrelated:
    5e-3 and 7e-3 of a gradient's norm; twice that is the bar."""
    model = example.GatedTokenModel(V, d, F, L, 3, rows=n * S + 5, act=act)
    teacher = torch.randn(V, 3, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    ids, y, _ = example.texts(n, S, V, 3, 0.0, 4, teacher)
    losses, dl = example.cross_entropy(model.forward(ids), y)
    model.backward(ids, dl / n)
    p = [t.double().clone().requires_grad_() for t in model.views(model.theta16)] + [t.double().clone().requires_grad_() for t in model.views(model.theta)[2 * L:]]
    real = (ids != 0).double()
    x = p[2 * L][ids.long().view(-1)] * d ** 0.5 * real.view(-1, 1)
    for l in range(L):
        pre = x @ p[2 * l].t()
        g, u = pre[:, :F], pre[:, F:]
        a = g * torch.sigmoid(g) if act == "silu" else g * 0.5 * torch.erfc(-g / 2 ** 0.5)
        x = x + (a * u) @ p[2 * l + 1].t()
    pooled = (x.view(n, S, d) * (real / real.sum(1, keepdim=True))[..., None]).sum(1)
    want = torch.nn.functional.cross_entropy(pooled @ p[-1].t(), y)
    want.backward()
    assert abs(float(losses.double().mean()) - want.item()) < 1e-2
    for got, t in zip(model.grads, p):
        assert float((got.double() - t.grad).norm() / t.grad.norm()) < (1e-2 if L == 1 else 1.4e-2)


def test_it_learns(example):
    model, net = example.main(30)
    V, S, C = 2000, 40, 4
    teacher = torch.randn(V, C, device="cuda", generator=torch.Generator(device="cuda").manual_seed(9))
    ids, y, _ = example.texts(64, S, V, C, 0.0, 77, teacher)
    right = float((model.forward(ids, keep=False).argmax(1) == y).float().mean())
    assert right > 0.5                       # of four classes
    assert int(model.status) == 0 and np.isfinite(float(model.norm[0]))
    assert all(bool(torch.isfinite(q).all()) for q in net.p)


def test_the_weights_tell_wrong_labels(example):
    """30 % of the training labels are wrong: the net has to give such texts less weight, and the rest more than half."""
    model, net = example.main(150)
    teacher = torch.randn(2000, 4, device="cuda", generator=torch.Generator(device="cuda").manual_seed(9))
    ids, y, flip = example.texts(64, 40, 2000, 4, 0.3, 78, teacher)
    w = net(example.cross_entropy(model.forward(ids, keep=False), y)[0])
    assert float(w[~flip].mean()) > 0.5 and float(w[flip].mean()) < float(w[~flip].mean()) - 0.1
