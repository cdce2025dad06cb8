"""optim.AdamW up to its library calls: what it refuses, what it hands over, its hooks.  No GPU: the tensors only say that
they are on one, and the library calls are recorded."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

import paper_2209_13258_b200.binding as B                                     # noqa: E402
from paper_2209_13258_b200 import optim                                        # noqa: E402
from test_modules_host import OnGpu, gpu                                       # noqa: E402


@pytest.fixture(autouse=True)
def calls(monkeypatch):
    """The tables that reach the step, one list of (param, grad, numel) per call."""
    seen = []
    zeros = torch.zeros

    def step(table, n, *a, **k):
        t = (B.AdamWTensor * max(n, 1)).from_address(table)
        seen.append([(e.param, e.grad, e.numel) for e in t[:n]])

    monkeypatch.setattr(B, "osdp_adamw_step", step)
    monkeypatch.setattr(B, "osdp_grad_norm", lambda *a, **k: None)
    monkeypatch.setattr(torch, "zeros", lambda *a, device=None, **k: gpu(zeros(*a, **k)))
    monkeypatch.setattr(B, "new_workspace", lambda n, device=None: zeros(n, dtype=torch.uint8))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(optim, "_DEVICE", lambda t: t.get_device())
    return seen


def make(*sizes, dtype=torch.float32, **kw):
    ps = [torch.nn.Parameter(gpu(torch.ones(n, dtype=dtype))) for n in sizes]
    for p in ps:
        p.grad = gpu(torch.ones(p.shape, dtype=dtype))
    return ps, optim.AdamW(ps, **kw)


def test_the_table_of_a_step(calls):
    ps, opt = make(100, 300)
    assert isinstance(ps[0], OnGpu)
    opt.step()
    assert calls == [[(p.data_ptr(), p.grad.data_ptr(), p.numel()) for p in ps]] and opt.steps == 1


@pytest.mark.parametrize("max_norm", [None, 1.0])
@pytest.mark.parametrize("change,error", [
    (lambda p: gpu(p.detach()[:50].clone()), ValueError), (lambda p: gpu(torch.ones(500)), ValueError),
    (lambda p: gpu(torch.ones(1)).expand(300), ValueError), (lambda p: gpu(torch.ones(600))[::2], ValueError),
    (lambda p: p.detach()[:50], ValueError), (lambda p: torch.ones(300).as_subclass(torch.Tensor), RuntimeError),
    (lambda p: gpu(torch.ones(300, dtype=torch.float64)), TypeError)])
def test_a_parameter_that_became_another_is_refused(calls, change, error, max_norm):
    ps, opt = make(100, 300, max_norm=max_norm)
    opt.step()
    new = change(ps[1])
    if type(new) is torch.Tensor:                     # as module.cpu() leaves it
        ps[1].__class__ = torch.nn.Parameter
    ps[1].data = new
    with pytest.raises(error, match="parameter 1"):
        opt.step()
    assert len(calls) == 1 and opt.steps == 1


@pytest.mark.parametrize("change,error", [(lambda g: gpu(torch.ones(50)), ValueError), (lambda g: g.detach()[:299], ValueError),
                                          (lambda g: gpu(torch.ones(300, dtype=torch.bfloat16)), TypeError)])
def test_a_gradient_that_does_not_fit_is_refused(calls, change, error):
    ps, opt = make(100, 300)
    opt.step()
    ps[1].grad.data = change(ps[1].grad)
    with pytest.raises(error, match="gradient 1"):
        opt.step()
    assert len(calls) == 1 and opt.steps == 1


def test_a_parameter_that_moved_in_memory_is_followed(calls):
    ps, opt = make(100, 300)
    opt.step()
    ps[1].data = gpu(torch.full((300,), 2.0))
    ps[0].grad = None
    opt.step()
    assert calls[1] == [(ps[1].data_ptr(), ps[1].grad.data_ptr(), 300)]
