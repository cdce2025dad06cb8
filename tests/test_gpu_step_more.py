"""AdamW around its kernel: parameters that change outside the step, small second moments, 8-bit states that have to follow,
norms over several optimisers and ranks.  Tolerances as in test_gpu_step.py where nothing else is said.
"""
import math

import pytest

from test_gpu_step import P, gen, half_unit, make, states, step64  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F64, QB = torch.float64, 256


# ---- masters and parameters

SIZES = [1, 255, 1000, 70001]


def check_step_from(before, ps, opt, t, lr, m, v):
    """One step from the fp32 values `before`, moments zero or as given."""
    for i, (p, o) in enumerate(zip(ps, opt.offsets)):
        want, _, _, upd = step64(before[i].double(), p.grad.double(), m[i], v[i], t, lr, 0.9, 0.999, 1e-8, 0.0)
        got = opt.master[o:o + p.numel()].double()
        assert bool(((got - want).abs() <= 4 * 2.0 ** -24 * before[i].double().abs() + 2.0 ** -20 * upd.abs() + 1e-30).all())
        assert torch.equal(p.detach(), got.bfloat16())


@pytest.mark.parametrize("how", ["in_place", "state_dict", "new_data", "data_and_refresh"])
def test_masters_follow_weights_that_change_outside_the_step(P, how):
    from paper_2209_13258_b200.optim import AdamW
    ps = make(SIZES, torch.bfloat16, 3)
    module = torch.nn.ParameterList(ps)
    opt = AdamW(ps, lr=1e-3, weight_decay=0.0, master=True)
    opt.step()
    new = [(p.detach() * 3 + 1).clone() for p in ps]
    m, v = zip(*[states(opt, i) for i in range(len(ps))])
    m, v = [t.clone() for t in m], [t.clone() for t in v]
    if how == "in_place":
        with torch.no_grad():
            for p, w in zip(ps, new):
                p.copy_(w)
    elif how == "state_dict":
        module.load_state_dict({str(i): w for i, w in enumerate(new)})
    elif how == "new_data":
        for p, w in zip(ps, new):
            p.data = w.clone()
    else:
        for p, w in zip(ps, new):
            p.data.copy_(w)
        opt.refresh_masters()
    opt.step()
    check_step_from([w.float() for w in new], ps, opt, 2, 1e-3, m, v)


def test_masters_keep_their_digits_where_nothing_changed(P):
    from paper_2209_13258_b200.optim import AdamW
    ps = make(SIZES, torch.bfloat16, 4)
    opt = AdamW(ps, lr=1e-3, weight_decay=0.0, master=True)
    opt.step()
    keep = opt.master.clone()
    with torch.no_grad():
        for p in ps:
            p.mul_(1.0)
        ps[2][:10] = 7.0
    opt.refresh_masters()
    o = opt.offsets[2]
    assert bool((opt.master[o:o + 10] == 7.0).all())
    keep[o:o + 10] = 7.0
    assert torch.equal(opt.master, keep)
    assert bool((keep != keep.bfloat16().float()).any())      # there are digits to lose


def test_masters_of_a_loaded_state_are_taken_as_they_are(P):
    from paper_2209_13258_b200.optim import AdamW
    a = make(SIZES, torch.bfloat16, 5)
    opt = AdamW(a, lr=1e-3, master=True)
    opt.step()
    b = make(SIZES, torch.bfloat16, 6)
    other = AdamW(b, lr=1e-3, master=True)
    for order in (0, 1):
        for k in (order, 1 - order):
            if k == 0:
                with torch.no_grad():
                    for p, q in zip(a, b):
                        q.copy_(p)
                        q.grad = p.grad.clone()
            else:
                other.load_state_dict(opt.state_dict())
        opt.step()
        other.step()
        assert torch.equal(opt.master, other.master) and all(torch.equal(p, q) for p, q in zip(a, b))
