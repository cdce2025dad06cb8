"""What the modules refuse before any address reaches a kernel.  No GPU: the tensors only say that they are
on one, and a library call fails the test."""
import pytest

torch = pytest.importorskip("torch")

import paper_2209_13258_b200.binding as B                                     # noqa: E402
from paper_2209_13258_b200 import nn as pnn                                    # noqa: E402

BF16, CUDA0 = torch.bfloat16, torch.device("cuda", 0)


class OnGpu(torch.Tensor):
    """A CPU tensor that gives itself out as one on cuda:0."""
    is_cuda = property(lambda self: True)
    device = property(lambda self: CUDA0)
    get_device = lambda self: 0                                                # noqa: E731


def gpu(t):
    return t.as_subclass(OnGpu)


def to_gpu(module):
    """The module's parameters and buffers say that they are on cuda:0."""
    for group in (module._parameters, module._buffers):
        for k, v in group.items():
            if v is not None:
                group[k] = torch.nn.Parameter(gpu(v.data)) if isinstance(v, torch.nn.Parameter) else gpu(v)
    return module


@pytest.fixture(autouse=True)
def no_kernel(monkeypatch):
    def reached(name):
        def call(*a, **k):
            raise AssertionError("%s was reached" % name)
        return call
    for name in ("osdp_block_norm_fwd", "osdp_split_linear_fwd_i8", "osdp_quantize_rows_i8", "osdp_split_linear_fwd", "osdp_split_mlp_fwd"):
        monkeypatch.setattr(B, name, reached(name))
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: torch.zeros(*a, **k))
    monkeypatch.setattr(torch, "empty_like", lambda t: torch.zeros(t.shape, dtype=t.dtype))
    monkeypatch.setattr(B, "new_workspace", lambda n, device=None: torch.zeros(n, dtype=torch.uint8))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(B, "_stream", lambda s: 0)


def norm(**kw):
    return pnn.ResidualNorm(64, post="layer", pre="layer", device="cpu", **kw)


def int8(bias=True):
    return pnn.Int8Linear(torch.ones(32, 64, dtype=torch.int8), torch.ones(32), torch.zeros(32) if bias else None)


X = torch.ones(4, 64, dtype=BF16)


@pytest.mark.parametrize("dtype", [BF16, torch.float16, torch.float64])
def test_a_cast_norm_is_refused(dtype):
    m = to_gpu(norm().to(dtype))
    for call in (lambda: m(gpu(X), gpu(X)), lambda: m(gpu(X)), lambda: m.forward_int8(gpu(X), gpu(X))):
        with torch.no_grad(), pytest.raises(TypeError, match="fp32"):
            call()


@pytest.mark.parametrize("name", ["w_post", "b_post", "gate", "w_pre", "b_pre"])
def test_each_vector_of_a_norm_is_looked_at(name):
    for other, error in ((torch.ones(64, dtype=BF16), TypeError), (torch.ones(56), ValueError), (torch.ones(128)[::2], ValueError)):
        m = to_gpu(norm())
        m._parameters[name] = torch.nn.Parameter(gpu(other))
        with torch.no_grad(), pytest.raises(error, match=name):
            m(gpu(X), gpu(X))
    m = to_gpu(norm())
    m._parameters[name] = torch.nn.Parameter(torch.ones(64))
    with torch.no_grad(), pytest.raises(RuntimeError, match="device"):
        m(gpu(X), gpu(X))


def test_a_norm_with_its_inputs_on_two_devices_is_refused():
    with torch.no_grad(), pytest.raises(RuntimeError, match="device"):
        to_gpu(norm())(gpu(X), X)


@pytest.mark.parametrize("dtype", [BF16, torch.float16])
def test_a_cast_int8_layer_is_refused(dtype):
    for bias in (True, False):
        with pytest.raises(TypeError, match="fp32"):
            to_gpu(int8(bias).to(dtype))(gpu(X))


def test_an_int8_layer_elsewhere_is_refused():
    codes, scale = X.to(torch.int8), torch.ones(4)
    with pytest.raises(RuntimeError, match="device"):
        int8()(gpu(X))
    for name in ("w_scale", "bias", "weight8"):
        m = to_gpu(int8())
        m._buffers[name] = m._buffers[name].clone().as_subclass(torch.Tensor)
        with pytest.raises(RuntimeError, match="device"):
            m(gpu(X))
    with pytest.raises(RuntimeError, match="device"):
        to_gpu(int8())((gpu(codes), scale))


def split_layers():
    return [pnn.SplitLinear(64, 32, device="cpu"), pnn.SplitMLP(64, 128, device="cpu")]


@pytest.mark.parametrize("dtype", [BF16, torch.float16, torch.float32])
def test_a_cast_split_layer_is_refused(dtype):
    """bf16 flat weights beside fp32 biases: any cast of the whole module spoils one of them."""
    for m in split_layers():
        with torch.no_grad(), pytest.raises(TypeError, match="has to be (fp32|bf16)"):
            to_gpu(m.to(dtype))(gpu(X))


def test_a_split_layer_elsewhere_is_refused():
    for m in split_layers():
        with torch.no_grad(), pytest.raises(RuntimeError, match="device"):
            m(gpu(X))
        for name in [k for k in m._parameters if m._parameters[k] is not None]:
            m2 = to_gpu(type(m)(64, 128, device="cpu"))
            m2._parameters[name] = torch.nn.Parameter(m._parameters[name].data.clone().resize_(m2._parameters[name].shape))
            with torch.no_grad(), pytest.raises(RuntimeError, match="device"):
                m2(gpu(X))


def test_what_is_right_reaches_the_kernel():
    for call in (lambda: to_gpu(split_layers()[0])(gpu(X)), lambda: to_gpu(split_layers()[1])(gpu(X)),
                 lambda: to_gpu(norm())(gpu(X), gpu(X)), lambda: to_gpu(int8())(gpu(X)), lambda: to_gpu(int8())((gpu(X.to(torch.int8)), gpu(torch.ones(4))))):
        with torch.no_grad(), pytest.raises(AssertionError, match="reached"):
            call()


def test_an_int8_layer_keeps_no_memory_of_its_calls(monkeypatch):
    """Codes and scales of a call's tokens are the call's: what the layer keeps does not depend on how many came (a captured
    graph would keep the address of what a later call replaces, and two streams would share it)."""
    kept, seen = [], []
    monkeypatch.setattr(B, "osdp_quantize_rows_i8", lambda x, M, K, q, s, *a, **k: seen.append(q))
    monkeypatch.setattr(B, "osdp_split_linear_fwd_i8", lambda *a, **k: kept.append(a[13]))
    m = to_gpu(int8())
    before = {k: v.data_ptr() for k, v in m._buffers.items() if v is not None}
    for tokens in (4, 300, 2):
        m(gpu(torch.ones(tokens, 64, dtype=BF16)))
    assert len(seen) == 3
    assert all(w.numel() == 256 and w.data_ptr() == kept[0].data_ptr() for w in kept)
    assert before == {k: v.data_ptr() for k, v in m._buffers.items() if v is not None}
    assert not [k for k, v in vars(m).items() if torch.is_tensor(v)]


def test_a_norm_keeps_no_memory_of_its_calls(monkeypatch):
    """The partial sums of a backward call are the call's: two streams would share what the module keeps."""
    used = []
    monkeypatch.setattr(B, "osdp_block_norm_fwd", lambda *a, **k: None)
    monkeypatch.setattr(B, "osdp_block_norm_bwd", lambda *a, **k: used.append(a[23]))
    m = to_gpu(norm())
    for tokens in (4, 300):
        x = gpu(torch.ones(tokens, 64, dtype=BF16)).requires_grad_(True)
        r, u = m(x, x)
        (r.sum() + u.sum()).backward()
    assert len(used) == 2 and used[0].numel() == used[1].numel() == B.osdp_block_norm_workspace_bytes(300, 64)[1]
    assert used[0].data_ptr() != used[1].data_ptr()
    assert not [k for k, v in vars(m).items() if torch.is_tensor(v)]


def test_calls_launch_on_their_tensors_device(monkeypatch):
    """The current device is another one: its current stream must not get the launch."""
    now, at = [1], []

    class Device:
        def __init__(self, device):
            self.index = torch.device(device).index

        def __enter__(self):
            self.old, now[0] = now[0], self.index

        def __exit__(self, *a):
            now[0] = self.old

    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", Device)
    for name in ("osdp_block_norm_fwd", "osdp_split_linear_fwd_i8", "osdp_quantize_rows_i8"):
        monkeypatch.setattr(B, name, lambda *a, **k: at.append(now[0]))
    with torch.no_grad():
        to_gpu(norm())(gpu(X), gpu(X))
        to_gpu(norm()).forward_int8(gpu(X), gpu(X))
        to_gpu(int8())(gpu(X))
        pnn.quantize_int8(gpu(X))
    assert at == [0] * 5 and now == [1]


@pytest.mark.parametrize("pre", [None, "rms"])
def test_outputs_of_a_norm_can_be_changed_in_place(monkeypatch, pre):
    """Under autograd too.  r is an input of the norm behind it, so a change before that norm's backward is reported there
    (by torch's version count); behind the last block nothing needs it."""
    monkeypatch.setattr(B, "osdp_block_norm_fwd", lambda *a, **k: None)
    monkeypatch.setattr(B, "osdp_block_norm_bwd", lambda *a, **k: None)
    m = to_gpu(pnn.ResidualNorm(64, post="rms", pre=pre, device="cpu"))
    x = gpu(torch.ones(2, 3, 64, dtype=BF16)).requires_grad_(True)
    r, u = m(x, x)
    assert r.shape == x.shape and r.is_contiguous()
    if pre:
        u.mul_(2.0)
        u.sum().backward(retain_graph=True)
    r.add_(1.0)
    if pre:
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            r.sum().backward()
    else:
        r.sum().backward()


def test_second_derivatives_are_refused(monkeypatch):
    """The backward passes are the library's calls, which autograd cannot differentiate: without the refusal the gradient of a
    gradient came out as if it did not depend on anything."""
    for name in ("osdp_block_norm_fwd", "osdp_block_norm_bwd", "osdp_split_linear_fwd", "osdp_split_linear_bwd", "osdp_split_mlp_fwd", "osdp_split_mlp_bwd"):
        monkeypatch.setattr(B, name, lambda *a, **k: None)
    monkeypatch.setattr(torch, "zeros_like", lambda t: torch.zeros(t.shape, dtype=t.dtype))
    calls = [(to_gpu(norm()), lambda m, x: m(x, x)[0])] + [(to_gpu(m), lambda m, x: m(x)) for m in split_layers()]
    for m, call in calls:
        x = gpu(X.clone()).requires_grad_(True)
        (g,) = torch.autograd.grad(call(m, x).float().square().sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            g.float().square().sum().backward()


def test_a_backward_pass_through_int8_is_refused(monkeypatch):
    monkeypatch.setattr(B, "osdp_split_linear_fwd_i8", lambda *a, **k: None)
    monkeypatch.setattr(B, "osdp_quantize_rows_i8", lambda *a, **k: None)
    m = to_gpu(int8())
    x = gpu(X.clone()).requires_grad_(True)
    with pytest.raises(RuntimeError, match="no gradient"):
        (m(x) + x[..., :32]).sum().backward()
    with torch.no_grad():
        assert not m(x).requires_grad
    assert not m(gpu(X)).requires_grad and not m(x.detach()).requires_grad


def test_the_first_norm_in_int8_writes_no_copy_of_x(monkeypatch):
    written = []
    monkeypatch.setattr(B, "osdp_block_norm_fwd", lambda *a, **k: written.append(a[16]))
    x = gpu(X)
    assert to_gpu(norm()).forward_int8(x)[0] is x and written == [None]
    assert to_gpu(norm(alpha=0.5)).forward_int8(x)[0] is not x and written[1] is not None
    assert to_gpu(norm()).forward_int8(x, x)[0] is not x and written[2] is not None


def test_an_int8_layer_looks_at_lengths_and_layouts():
    """Buffers that a program has put in place of the layer's own."""
    for name, other in (("w_scale", torch.ones(1).expand(32)), ("bias", torch.ones(64)[::2]), ("w_scale", torch.ones(16)), ("bias", torch.ones(8))):
        m = to_gpu(int8())
        m._buffers[name] = gpu(other)
        with pytest.raises(ValueError, match=name):
            m(gpu(X))
    for other in (torch.ones(64, 32, dtype=torch.int8).t(), torch.ones(16, 64, dtype=torch.int8), torch.ones(1, 64, dtype=torch.int8).expand(32, 64)):
        m = to_gpu(int8())
        m._buffers["weight8"] = gpu(other)
        with pytest.raises(RuntimeError, match="weight8"):
            m(gpu(X))
