"""Router and mixture of experts as modules: a run of all operators together against the formulas in 64 bits."""
import math

import pytest
import torch

import paper_2209_13258_b200 as P
from paper_2209_13258_b200.nn import ExpertMLP, ExpertRouter
from paper_2209_13258_b200.optim import AdamW, ClippedStep

pytestmark = pytest.mark.gpu
D64, BF16 = torch.float64, torch.bfloat16
HALF16 = 2.0 ** -8


def gelu(z):
    return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))


def reference(x, weights, idx, w1, w2, b1, b2, act):
    """The definition, expert by expert."""
    out = torch.zeros_like(x)
    for e in range(w1.shape[0]):
        t, j = (idx == e).nonzero(as_tuple=True)
        z = x[t] @ w1[e].t() + (b1[e] if b1 is not None else 0.0)
        y = (gelu(z) if act else z) @ w2[e].t() + (b2[e] if b2 is not None else 0.0)
        out = out.index_add(0, t, y * weights[t, j][:, None])
    return out


def close(got, want, roundings):
    """Each of the chain's roundings to bf16 is off by HALF16 of its value at most; the sums over hundreds of them in a norm stay
    below the sum of the bounds."""
    return float((got.to(D64) - want).norm()) <= roundings * HALF16 * float(want.norm()) + 1e-30


@pytest.mark.parametrize("T,H,F,E,k,bias,act", [(1, 64, 128, 8, 2, True, True), (37, 72, 200, 5, 3, True, True), (600, 256, 512, 4, 2, True, True),
                                                (600, 256, 512, 16, 1, False, False), (2500, 512, 1024, 3, 2, True, True)])
def test_mixture_of_experts(T, H, F, E, k, bias, act):
    torch.manual_seed(T + E)
    router = ExpertRouter(E, k, scale=1.5)
    mlp = ExpertMLP(H, F, E, bias=bias, act=P.ACT_GELU_TANH if act else P.ACT_NONE)
    with torch.no_grad():
        mlp.flat_param.copy_(torch.randn_like(mlp.flat_param) * H ** -0.5)
        if bias:
            mlp.b1.normal_(std=0.2)
            mlp.b2.normal_(std=0.2)
    x = torch.randn(T, H, device="cuda").to(BF16).requires_grad_()
    logits = torch.randn(T, E, device="cuda").requires_grad_()
    dout = torch.randn(T, H, device="cuda").to(BF16)
    weights, idx = router(logits)
    out = mlp(x, weights, idx)
    out.backward(dout)
    wide = lambda v: v.detach().to(D64).requires_grad_() if v is not None else None      # noqa: E731
    x64, l64, w1, w2, b1, b2 = wide(x), wide(logits), wide(mlp.w1), wide(mlp.w2), wide(mlp.b1), wide(mlp.b2)
    s = torch.softmax(l64, 1).gather(1, idx.long())
    want = reference(x64, 1.5 * s / s.sum(1, keepdim=True), idx.long(), w1, w2, b1, b2, act)
    want.backward(dout.to(D64))
    assert close(out.detach(), want.detach(), 4)                       # h, y, out, and the approximate tanh
    n = H * F * E
    grads = {"x": (x.grad, x64.grad, 6), "logits": (logits.grad, l64.grad, 6), "w1": (mlp.flat_param.grad[:n].view_as(w1), w1.grad, 6),
             "w2": (mlp.flat_param.grad[n:].view_as(w2), w2.grad, 5)}
    if bias:
        grads |= {"b1": (mlp.b1.grad, b1.grad, 5), "b2": (mlp.b2.grad, b2.grad, 2)}
    if k == 1:       # the only weight of a token is the scale: its gradient is rounding alone
        assert float(logits.grad.abs().max()) <= 1e-3 * float(dout.to(D64).norm())
        del grads["logits"]
    for name, (a, b, roundings) in grads.items():
        assert close(a, b, roundings), name


def test_gradient_of_the_loss_against_differences():
    """Along random directions of every input: the change of the loss and its gradient's prediction."""
    torch.manual_seed(5)
    T, H, F, E, k = 64, 64, 128, 4, 2
    mlp, router = ExpertMLP(H, F, E), ExpertRouter(E, k, score="sigmoid")
    with torch.no_grad():
        mlp.flat_param.copy_(torch.randn_like(mlp.flat_param) * H ** -0.5)
    x = torch.randn(T, H, device="cuda").to(BF16).requires_grad_()
    logits = torch.randn(T, E, device="cuda").requires_grad_()
    weights, idx = router(logits)
    out = mlp(x, weights, idx)
    target = torch.randn(T, H, device="cuda", dtype=D64)
    (out.float() * target.float()).sum().backward()

    def loss(dx, dl, dw):
        s = torch.sigmoid(logits.detach().to(D64) + dl).gather(1, idx.long())
        flat = mlp.flat_param.detach().to(D64) + dw
        n = E * H * F
        o = reference(x.detach().to(D64) + dx, s / s.sum(1, keepdim=True), idx.long(), flat[:n].view(E, F, H), flat[n:].view(E, H, F), None, None, True)
        return float((o * target).sum())
    for turn in range(3):
        h = 1e-4
        d = [torch.randn_like(v, dtype=D64) for v in (x, logits, mlp.flat_param)]
        for i, (v, dv) in enumerate(zip((x, logits, mlp.flat_param), d)):
            step = [dv * h if j == i else torch.zeros_like(d[j]) for j in range(3)]
            diff = (loss(*step) - loss(*[-s for s in step])) / (2 * h)
            pred = float((v.grad.to(D64) * dv).sum())
            # the gradient is off by some roundings of its norm, and a random direction sees that times its own spread
            assert abs(diff - pred) <= 6 * HALF16 * 4 * float(v.grad.to(D64).norm()) + 1e-5 * abs(diff)


def test_router_options_and_shapes():
    torch.manual_seed(6)
    r = ExpertRouter(32, 4, score="sigmoid", groups=8, top_groups=2, group_take=2, bias=True, scale=2.0)
    r.bias.normal_(std=0.3)
    logits = torch.randn(3, 50, 64, device="cuda")[..., 16:48].requires_grad_()
    w, idx = r(logits)
    assert w.shape == idx.shape == (3, 50, 4) and idx.dtype == torch.int32 and not idx.requires_grad
    assert torch.allclose(w.sum(-1), torch.full_like(w[..., 0], 2.0), atol=1e-5)
    assert int(torch.tensor([len(set((row // 4).tolist())) for row in idx.view(-1, 4)]).max()) <= 2
    again = r(logits.detach().contiguous())
    assert torch.equal(again[0], w) and torch.equal(again[1], idx)
    (w * torch.randn_like(w)).sum().backward(retain_graph=True)
    with pytest.raises(RuntimeError):           # a second derivative is refused
        g, = torch.autograd.grad((w * w.detach()).sum(), [logits], create_graph=True)
        g.sum().backward()
    r16 = ExpertRouter(32, 4)
    assert r16(torch.randn(7, 32, device="cuda").bfloat16())[0].dtype == torch.float32
    with pytest.raises(TypeError):
        r16(torch.randn(7, 32, device="cuda").half())
    with pytest.raises(ValueError):
        r16(torch.randn(7, 31, device="cuda"))
    with pytest.raises(TypeError):
        ExpertRouter(32, 4, bias=True).bfloat16()(torch.randn(7, 32, device="cuda"))


def test_mlp_refuses():
    m = ExpertMLP(64, 64, 4)
    x, w, i = torch.randn(5, 64, device="cuda").bfloat16(), torch.rand(5, 2, device="cuda"), torch.zeros(5, 2, dtype=torch.int32, device="cuda")
    for args, error in (((x.float(), w, i), TypeError), ((x, w.bfloat16(), i), TypeError), ((x, w, i.long()), TypeError), ((x[:, :32], w, i), ValueError),
                        ((x, w[:4], i[:4]), ValueError), ((x, w, i[:, :1]), ValueError), ((x, w.cpu(), i), RuntimeError), ((x, w, i.cpu()), RuntimeError)):
        with pytest.raises(error):
            m(*args)
    with pytest.raises(TypeError):
        ExpertMLP(64, 64, 4).float()(x, w, i)
    with pytest.raises(TypeError):
        ExpertMLP(64, 64, 4).bfloat16()(x, w, i)


def test_parts_without_a_gradient_shapes_and_no_tokens():
    torch.manual_seed(7)
    m = ExpertMLP(64, 128, 4)
    x, w = torch.randn(2, 9, 64, device="cuda").bfloat16(), torch.rand(2, 9, 2, device="cuda")
    i = torch.randint(0, 4, (2, 9, 2), device="cuda").to(torch.int32)
    full = m(x.clone().requires_grad_(), w.clone().requires_grad_(), i)
    with torch.no_grad():
        assert torch.equal(m(x, w, i), full) and full.shape == x.shape
    for on in ("x", "w", "flat_param", "b1", "b2"):
        xs, ws = x.clone().requires_grad_(on == "x"), w.clone().requires_grad_(on == "w")
        for n, p in m.named_parameters():
            p.requires_grad_(n == on)
            p.grad = None
        m(xs, ws, i).float().sum().backward()
        got = {"x": xs.grad, "w": ws.grad} | {n: p.grad for n, p in m.named_parameters()}
        assert got[on] is not None and bool(got[on].float().abs().sum() > 0) and all(v is None for n, v in got.items() if n != on)
    for p in m.parameters():
        p.requires_grad_(True)
    none = torch.empty(0, 64, device="cuda", dtype=BF16, requires_grad=True)
    out = m(none, torch.empty(0, 2, device="cuda"), torch.empty(0, 2, dtype=torch.int32, device="cuda"))
    m.flat_param.grad = None
    out.sum().backward()
    assert out.shape == (0, 64) and bool((m.flat_param.grad == 0).all())
    # choices of nobody, rows that come in parts of a wider tensor
    wide = torch.randn(9, 128, device="cuda").bfloat16()
    i2 = torch.full((9, 2), -1, dtype=torch.int32, device="cuda")
    assert bool((m(wide[:, 64:], torch.rand(9, 2, device="cuda"), i2) == 0).all())


def test_streams_and_captured_training_step():
    torch.manual_seed(8)
    m, r = ExpertMLP(64, 128, 8), ExpertRouter(8, 2)
    with torch.no_grad():
        m.flat_param.copy_(torch.randn_like(m.flat_param) * 0.1)
    data = [(torch.randn(300, 64, device="cuda").bfloat16(), torch.randn(300, 8, device="cuda")) for _ in range(4)]
    torch.cuda.synchronize()

    def step(x, l):
        x, l = x.detach().requires_grad_(), l.detach().requires_grad_()
        out = m(x, *r(l))
        # (the graph is let go: one that lives on the same parameters while another is captured is torch's own stumbling block)
        return (out.detach(),) + torch.autograd.grad(out.float().square().sum(), [x, l, m.flat_param, m.b1, m.b2])
    want = [step(*d) for d in data]
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    got = []
    for s, d in zip(streams, data):
        with torch.cuda.stream(s):
            got.append(step(*d))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(u, v) for u, v in zip(a, b))
    # captured once, replayed on other data
    x, l = data[0][0].clone(), data[0][1].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(x, l)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step(x, l)
    for d, w in zip(data, want):
        x.copy_(d[0])
        l.copy_(d[1])
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(out, w))
    del g


def test_training_with_the_optimiser():
    """Gradients reach every parameter, and a step changes them."""
    torch.manual_seed(9)
    m, r = ExpertMLP(64, 128, 4), ExpertRouter(4, 2)
    gate = torch.nn.Linear(64, 4, device="cuda")
    opt = ClippedStep([AdamW([m.flat_param], lr=1e-2, state_dtype="e4m3", master=True), AdamW([m.b1, m.b2, *gate.parameters()], lr=1e-2)], max_norm=1.0)
    x = torch.randn(200, 64, device="cuda")
    before = [p.detach().clone() for p in (*m.parameters(), *gate.parameters())]
    (m(x.bfloat16(), *r(gate(x))).float() - x).square().mean().backward()
    for p in (*m.parameters(), *gate.parameters()):
        assert p.grad is not None and bool(torch.isfinite(p.grad).all()) and bool(p.grad.float().abs().max() > 0)
    opt.step()
    assert all(not torch.equal(a, b) for a, b in zip(before, (*m.parameters(), *gate.parameters())))


def test_example_with_experts():
    """It runs, and gradients reach every parameter."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import residual_blocks
    losses, _ = residual_blocks.main(["--hidden", "128", "--ffn", "256", "--blocks", "2", "--tokens", "300", "--steps", "3", "--experts", "6"])
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses)
    net = residual_blocks.Stack(128, 256, 2, experts=6)
    net(torch.randn(300, 128, device="cuda")).square().mean().backward()
    for n, p in net.named_parameters():
        assert p.grad is not None and bool(torch.isfinite(p.grad).all()) and bool(p.grad.float().abs().max() > 0), n
