"""What the mixture-of-experts modules keep between forward and backward."""
import pytest
import torch

import paper_2209_13258_b200 as P
from paper_2209_13258_b200.nn import ExpertMLP, ExpertRouter

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def batch(T=60, H=64, E=4, k=2, grad=True):
    x = torch.randn(T, H, device="cuda").to(BF16).requires_grad_(grad)
    return x, torch.rand(T, k, device="cuda").requires_grad_(grad), torch.randint(0, E, (T, k), device="cuda").to(torch.int32)


@pytest.mark.parametrize("change", [{"scale": 3.0}, {"renormalise": False}, {"score": P.SCORE_SOFTMAX}, {"top_k": 1}])
def test_a_router_changed_after_the_forward(change):
    """The gradient is that of what the forward did."""
    torch.manual_seed(1)
    logits, dw = torch.randn(100, 16, device="cuda"), torch.randn(100, 3, device="cuda")
    grads = []
    for later in ({}, change):
        r, l = ExpertRouter(16, 3, score="sigmoid", scale=1.5), logits.clone().requires_grad_()
        w, _ = r(l)
        for name, v in later.items():
            setattr(r, name, v)
        w.backward(dw)
        grads.append(l.grad)
    assert torch.equal(*grads)


def test_an_activation_changed_after_the_forward():
    torch.manual_seed(2)
    m = ExpertMLP(64, 128, 4)
    x, w, i = batch()
    grads = []
    for act in (P.ACT_GELU_TANH, P.ACT_GELU_ERF):
        m.act = P.ACT_GELU_TANH
        out = m(x, w, i)
        m.act = act
        grads.append(torch.autograd.grad(out.float().square().sum(), [x, w, m.flat_param]))
    assert all(torch.equal(a, b) for a, b in zip(*grads))
