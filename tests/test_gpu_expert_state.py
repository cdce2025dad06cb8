"""What the mixture-of-experts modules keep between forward and backward, and what is left of a wait that ran out."""
import pytest
import torch

import paper_2209_13258_b200 as P
from paper_2209_13258_b200 import binding as B
from paper_2209_13258_b200.nn import ExpertMLP, ExpertRouter

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
TIMEOUT = 8


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


def kept(m, *args):
    """Bytes of what the forward keeps for the backward, inputs and parameters aside."""
    seen = {}
    known = {t.untyped_storage().data_ptr() for t in (*args, *m.parameters())}

    def pack(t):
        if t.untyped_storage().data_ptr() not in known:
            seen[t.untyped_storage().data_ptr()] = t.untyped_storage().nbytes()
        return t
    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t):
        out = m(*args)
    out.float().sum().backward()
    return sum(seen.values())


def test_only_what_the_gradients_need_is_kept():
    torch.manual_seed(3)
    m = ExpertMLP(64, 128, 4)
    x, w, i = batch(T=500)
    rows = P.osdp_expert_rows(500, 2, 4)[1]
    whole = kept(m, x, w, i)
    assert whole - kept(m, x, w.detach(), i) == rows * 64 * 2               # the combined rows: the gradient of the weights
    m.flat_param.requires_grad_(False)
    assert whole - kept(m, x, w, i) == rows * (64 + 128) * 2                # both products' rows: the experts' gradients
    assert x.grad is not None and m.b1.grad is not None and m.flat_param.grad is not None


def test_a_larger_flat_buffer_has_a_gradient_of_zeros_behind_the_experts():
    torch.manual_seed(4)
    m = ExpertMLP(64, 128, 4)
    n = m.flat_param.numel()
    filled = torch.full((4 * n,), 7.0, dtype=BF16, device="cuda")      # what a new allocation may find
    del filled
    m.flat_param.data = torch.cat([m.flat_param.data, torch.ones(3 * n, dtype=BF16, device="cuda")])
    x, w, i = batch()
    m(x, w, i).float().sum().backward()
    assert m.flat_param.grad.shape == (4 * n,) and bool((m.flat_param.grad[n:] == 0).all()) and bool((m.flat_param.grad[:n] != 0).any())


def test_a_wait_that_runs_out_in_the_backward_leaves_its_trace(monkeypatch):
    """The module's status word has it, as it has the forward's; it is cleared by being read."""
    torch.manual_seed(5)
    m = ExpertMLP(64, 128, 4)
    x, w, i = batch()
    read = lambda: P.osdp_read_device_status(m._status)                                              # noqa: E731
    m(x, w, i).float().sum().backward()
    assert read() == (0, 0)
    call = B.osdp_expert_linear_bwd
    for which in (0, 1):                    # each of the backward's two products
        calls = []

        def broken(*args):
            rc = call(*args)
            if len(calls) == which:         # ws, stream, check come last
                P.osdp_debug_wait_probe(args[-3], 1000, args[-2])
            calls.append(rc)
            return rc
        monkeypatch.setattr(B, "osdp_expert_linear_bwd", broken)
        m(x, w, i).float().sum().backward()
        monkeypatch.setattr(B, "osdp_expert_linear_bwd", call)
        assert len(calls) == 2 and read() == (0, TIMEOUT) and read() == (0, 0)


def test_status_words_meet():
    a, b = P.new_workspace(256), P.new_workspace(256)
    P.osdp_join_status(a, b, check=True)
    assert P.osdp_read_device_status(b) == (0, 0)
    P.osdp_debug_wait_probe(a, 1000)
    P.osdp_join_status(a, b, check=True)
    P.osdp_join_status(P.new_workspace(256), b, check=True)          # one without a mark leaves the other's
    assert P.osdp_read_device_status(b) == (0, TIMEOUT) and P.osdp_read_device_status(a) == (0, TIMEOUT) and P.osdp_read_device_status(b) == (0, 0)
