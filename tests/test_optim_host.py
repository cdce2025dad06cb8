"""optim.AdamW up to its library calls: what it refuses, what it hands over, its hooks.  No GPU: the tensors only say that
they are on one, and the library calls are recorded."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

import paper_2209_13258_b200.binding as B                                     # noqa: E402
from paper_2209_13258_b200 import optim                                        # noqa: E402
from test_modules_host import OnGpu, gpu                                       # noqa: E402


def patch(monkeypatch):
    """Returns the list that gets the tables that reach the step, one list of (param, grad, numel) per call."""
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


@pytest.fixture(autouse=True)
def calls(monkeypatch):
    return patch(monkeypatch)


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


# ---- one norm over several optimisers and ranks

def fake_squares(monkeypatch, log=None):
    def squares(table, n, dtype, to, ws, **k):
        t = (B.AdamWTensor * max(n, 1)).from_address(table)
        c = {B.DTYPE_FP32: ctypes.c_float, B.DTYPE_BF16: ctypes.c_uint16}[dtype]
        total = 0.0
        for e in t[:n]:
            a = list((c * e.numel).from_address(e.grad))
            if dtype == B.DTYPE_BF16:
                a = torch.tensor(a, dtype=torch.int32).to(torch.uint16).view(torch.bfloat16).double().tolist()
            total += sum(v * v for v in a)
        ctypes.c_double.from_address(to).value = total

    def coefficient(sums, n, max_norm, out, **k):
        norm = float(sums[:n].sum()) ** 0.5
        out[0], out[1] = norm, min(1.0, max_norm / (norm + 1e-6))

    monkeypatch.setattr(B, "osdp_grad_squares", squares)
    monkeypatch.setattr(B, "osdp_clip_coefficient", coefficient)


class NoDevice:
    def __init__(self, *a):
        pass

    __enter__ = __exit__ = lambda self, *a: None                               # noqa: E731


def test_a_clipped_step_hands_one_coefficient_to_all(calls, monkeypatch):
    fake_squares(monkeypatch)
    monkeypatch.setattr(torch.cuda, "device", NoDevice)
    clips = []
    monkeypatch.setattr(B, "osdp_adamw_step", lambda *a, **k: clips.append(a[13]))
    _, a = make(100, 300)
    _, b = make(50, dtype=torch.bfloat16)
    c = optim.ClippedStep([a, b], max_norm=2.0)
    c.step()
    assert abs(float(c.grad_norm[0]) - 450 ** 0.5) < 1e-5
    assert len(clips) == 2 and all(v is c.grad_norm for v in clips)
    a.step()
    assert clips[2] is None            # by itself an optimiser does not clip


def test_a_clipped_step_refuses():
    _, a = make(100)
    _, own = make(100, max_norm=1.0)
    ps, _ = make(100)
    shard = optim.AdamW([{"params": ps, "sharded": True}])
    with pytest.raises(ValueError, match="max_norm"):
        optim.ClippedStep([a, own], 1.0)
    with pytest.raises(ValueError, match="comm"):
        optim.ClippedStep([a, shard], 1.0)
    with pytest.raises(TypeError):
        optim.ClippedStep([], 1.0)
    with pytest.raises(TypeError):
        optim.ClippedStep([a, torch.optim.SGD([torch.nn.Parameter(torch.ones(1))], lr=1.0)], 1.0)


WORKER = """
import os, sys
sys.path[:0] = [%r, %r]
import pytest, torch, torch.distributed as dist
import test_optim_host as T
from test_modules_host import gpu
from paper_2209_13258_b200 import binding as B, optim
from paper_2209_13258_b200.zdp import DistComm
dist.init_process_group("gloo")
rank = dist.get_rank()
mp = pytest.MonkeyPatch()
T.patch(mp)
T.fake_squares(mp)
mp.setattr(torch.cuda, "device", T.NoDevice)
shard = torch.nn.Parameter(gpu(torch.ones(100)))
shard.grad = gpu(torch.full((100,), 3.0 if rank else 0.1))
both = torch.nn.Parameter(gpu(torch.ones(50)))
both.grad = gpu(torch.full((50,), 0.7))
half = torch.nn.Parameter(gpu(torch.ones(20, dtype=torch.bfloat16)))
half.grad = gpu(torch.full((20,), 0.5, dtype=torch.bfloat16))
c = optim.ClippedStep([optim.AdamW([{"params": [both]}, {"params": [shard], "sharded": True}]), optim.AdamW([half])], 1.0, comm=DistComm())
for _ in range(3):
    c.step()
    want = (100 * 9.0 + 100 * 0.1 ** 2 + 50 * 0.49 + 20 * 0.25) ** 0.5
    assert abs(float(c.grad_norm[0]) - want) < 1e-4 * want, (rank, c.grad_norm)
    print("rank", rank, c.grad_norm.tolist())
dist.barrier()
dist.destroy_process_group()
"""


def test_two_gloo_ranks_get_one_coefficient():
    import os
    import subprocess
    import sys
    here = os.path.dirname(os.path.abspath(__file__))
    procs = [subprocess.Popen([sys.executable, "-c", WORKER % (os.path.dirname(here), here)], stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True,
                              env=dict(os.environ, RANK=str(r), WORLD_SIZE="2", MASTER_ADDR="127.0.0.1", MASTER_PORT="29755")) for r in (0, 1)]
    outs = [p.communicate(timeout=180) for p in procs]
    for p, (_, err) in zip(procs, outs):
        assert p.returncode == 0, err[-3000:]
    lines = [[line.split("]")[0].split("[")[1] for line in o.splitlines() if line.startswith("rank")] for o, _ in outs]
    assert len(lines[0]) == 3 and lines[0] == lines[1]


def test_squares_and_coefficient_refuse():
    """The library's own checks stand before any launch: made-up addresses are never read."""
    A, need = 1 << 20, B.osdp_grad_norm_workspace_bytes(1)[1]
    t = (B.AdamWTensor * 1)()
    t[0].grad, t[0].numel = A, 100
    go = lambda t=t, n=1, dt=1, out=A, ws=(A, need): B.osdp_grad_squares(t, n, dt, out, ws, stream=0)          # noqa: E731
    assert [go(out=None), go(ws=None), go(ws=(A + 8, need)), go(ws=(A, 256)), go(dt=2), go(n=-1), go(out=A + 4)] == [1, 1, 4, 5, 6, 2, 4]
    co = lambda sums=A, n=2, mx=1.0, out=A: B.osdp_clip_coefficient(sums, n, mx, out, stream=0)                # noqa: E731
    assert [co(sums=None), co(out=None), co(n=-1), co(mx=float("nan")), co(sums=A + 4), co(out=A + 2)] == [1, 1, 2, 6, 4, 4]


# ---- torch's conventions

def test_hooks_are_called_as_torch_calls_them(calls):
    """Global and own hooks, in torch's order and with torch's arguments; a pre-hook may replace the arguments."""
    from torch.optim.optimizer import register_optimizer_step_post_hook, register_optimizer_step_pre_hook
    ps, opt = make(100)
    seen, ran = [], []
    closure = lambda: ran.append("given") or 1.0                               # noqa: E731
    other = lambda: ran.append("other") or 2.0                                 # noqa: E731
    handles = [register_optimizer_step_pre_hook(lambda o, a, k: seen.append(("global pre", o is opt, a, k))),
               register_optimizer_step_post_hook(lambda o, a, k: seen.append(("global post", o is opt, a, k))),
               opt.register_step_pre_hook(lambda o, a, k: seen.append(("pre", o is opt, a, k)) or ((o, other), k)),
               opt.register_step_post_hook(lambda o, a, k: seen.append(("post", o is opt, a, k)))]
    try:
        assert opt.step(closure) == 2.0
    finally:
        for h in handles:
            h.remove()
    assert ran == ["other"] and len(calls) == 1
    assert seen == [("global pre", True, (opt, closure), {}), ("pre", True, (opt, closure), {}), ("post", True, (opt, other), {}),
                    ("global post", True, (opt, other), {})]
    opt.register_step_pre_hook(lambda o, a, k: 3)
    with pytest.raises(RuntimeError):
        opt.step()


def test_a_step_shows_in_a_profile(calls):
    ps, opt = make(100)
    opt.step()
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CPU]) as prof:
        opt.step()
    assert any("Optimizer.step#AdamW" in e.key for e in prof.key_averages())


@pytest.mark.parametrize("name", ["osdp_adamw_step", "osdp_grad_norm"])
def test_a_step_that_the_library_refuses_is_not_counted(calls, monkeypatch, name):
    """The count sets the bias correction: a refused step (here: its betas) has not happened."""
    ps, opt = make(100, max_norm=1.0)
    opt.step()

    def refuse(*a, **k):
        raise B.OsdpError(6, name)

    with monkeypatch.context() as m:
        m.setattr(B, name, refuse)
        with pytest.raises(B.OsdpError):
            opt.step()
    assert opt.steps == 1
    opt.step()
    assert opt.steps == 2


def test_gradients_come_and_go(calls):
    """The look at what came last time must not take a missing gradient for one that fits."""
    ps, opt = make(100, 300)
    for want in ([0, 1], [0, 1], [0], [0, 1], [1], []):
        for i, p in enumerate(ps):
            p.grad = gpu(torch.ones(p.shape)) if i in want else None
        opt.step()
        assert [c[0] for c in calls[-1]] == [ps[i].data_ptr() for i in want]


def test_sharded_parameters_are_not_clipped_by_one_ranks_norm():
    ps, _ = make(100)
    with pytest.raises(ValueError, match="ClippedStep"):
        optim.AdamW([{"params": ps, "sharded": True}], max_norm=1.0)
    optim.AdamW([{"params": ps, "sharded": False}], max_norm=1.0)
