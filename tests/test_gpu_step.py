"""AdamW over many tensors (osdp_adamw_step, osdp_grad_norm, optim.AdamW) against the formulas in 64 bits.

Tolerances.  fp32 states: three roundings, 4 * 2^-24 of the terms' magnitudes.  fp32 parameters: two roundings of the
value and a relative 2^-20 of the update (its division is good to a few units in the last place, m and v to the above).
bf16 parameters: half a unit in the last place on top.  8-bit states: half a step of e4m3 (2^-4 of the value, 2^-10 of the scale
below the normal range) and 2e-6 for the fp32 arithmetic.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F64 = torch.float64
QB = 256


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2209_13258_b200 as pkg
    pkg.lib()
    return pkg


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *n: torch.randn(*n, device="cuda", generator=g)


def half_unit(v):
    """Half a unit in the last place of bf16 (8 significant bits) at |v|: what rounding to nearest may cost."""
    return torch.ldexp(torch.ones_like(v), torch.frexp(v.abs().clamp_min(1e-300))[1] - 9)


def make(sizes, dtype, seed, shift=0):
    """Parameters with gradients; `shift` elements in front of each, so that their addresses are only element-aligned."""
    rnd = gen(seed)
    ps = []
    for n in sizes:
        p = torch.nn.Parameter((rnd(n + shift) * 0.05).to(dtype)[shift:])
        p.grad = (rnd(n + shift) * 0.01 * (1 + len(ps) % 3)).to(dtype)[shift:]
        ps.append(p)
    return ps


def step64(w, g, m, v, t, lr, b1, b2, eps, wd, coef=1.0):
    g = g * coef
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    upd = lr / (1 - b1 ** t) * m / (v.sqrt() / math.sqrt(1 - b2 ** t) + eps)
    return w * (1 - lr * wd) - upd, m, v, upd


def states(opt, i):
    """fp64 m and v of parameter i as the optimiser holds them."""
    o, n = opt.offsets[i], opt._params[i].numel()
    if opt.exp_avg.dtype == torch.float32:
        return opt.exp_avg[o:o + n].double(), opt.exp_avg_sq[o:o + n].double()
    at = torch.arange(o, o + n, device="cuda") // QB
    m = opt.exp_avg[o:o + n].float().double() * opt.exp_avg_scale[at].double()
    r = opt.exp_avg_sq[o:o + n].float().double() * opt.exp_avg_sq_scale[at].double()
    return m, r * r


def half_step(value, scale):
    return torch.maximum(value.abs() * 2.0 ** -4, scale * 2.0 ** -10) * 1.0001 + 2e-6 * value.abs()


SIZES = [1, 7, 255, 256, 257, 4096, 4097, 30001, 8, 131072]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("state", ["fp32", "e4m3"])
@pytest.mark.parametrize("master", [False, True])
@pytest.mark.parametrize("shift", [0, 1])
def test_steps(P, dtype, state, master, shift):
    from paper_2209_13258_b200.optim import AdamW
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    if master and dt == torch.float32:
        with pytest.raises(ValueError):
            AdamW(make([8], dt, 1), master=True)
        return
    ps = make(SIZES, dt, 3, shift)
    lr, b1, b2, eps = 3e-3, 0.9, 0.97, 1e-8
    opt = AdamW([{"params": ps[:6], "weight_decay": 0.1}, {"params": ps[6:], "weight_decay": 0.0, "lr": 1e-3}], lr=lr, betas=(b1, b2), eps=eps,
                state_dtype=state, master=master)
    for t in (1, 2, 3):
        before = [((opt.master[o:o + p.numel()].double() if master else p.detach().double()), p.grad.double(), *states(opt, i))
                  for i, (p, o) in enumerate(zip(ps, opt.offsets))]
        opt.step()
        torch.cuda.synchronize()
        for i, (p, o) in enumerate(zip(ps, opt.offsets)):
            w, g, m, v = before[i]
            n = p.numel()
            rate, wd = (lr, 0.1) if i < 6 else (1e-3, 0.0)
            wr, mr, vr, upd = step64(w, g, m, v, t, rate, b1, b2, eps, wd)
            tol = 4 * 2.0 ** -24 * w.abs() + 2.0 ** -20 * upd.abs() + 1e-30
            if master:
                assert bool(((opt.master[o:o + n].double() - wr).abs() <= tol).all())
                assert torch.equal(p.detach(), opt.master[o:o + n].bfloat16())
            else:
                extra = half_unit(wr) if dt == torch.bfloat16 else 0.0
                assert bool(((p.detach().double() - wr).abs() <= tol + extra).all())
            mg, vg = states(opt, i)
            if state == "fp32":
                assert bool(((mg - mr).abs() <= 4 * 2.0 ** -24 * ((b1 * m).abs() + ((1 - b1) * g).abs()) + 1e-37).all())
                assert bool(((vg - vr).abs() <= 4 * 2.0 ** -24 * vr + 1e-37).all())
            else:
                at = torch.arange(o, o + n, device="cuda") // QB
                sm, sv = opt.exp_avg_scale[at].double(), opt.exp_avg_sq_scale[at].double()
                assert bool(((mg - mr).abs() <= half_step(mr, sm) + 1e-37).all())
                root, want = vg.sqrt(), vr.sqrt()
                lifted = (want > 0) & (want < sv * 2.0 ** -9)      # below the smallest code: kept there
                assert bool(((root - want).abs() <= torch.where(lifted, sv * 2.0 ** -9, half_step(want, sv)) + 1e-37).all())
                assert bool((root[want > 0] > 0).all())
        for s in (opt.exp_avg, opt.exp_avg_sq):                      # the padding of a tensor's last block stays zero
            flat = s.float()
            for p, o in zip(ps, opt.offsets):
                assert float(flat[o + p.numel():-(-(o + p.numel()) // QB) * QB].abs().sum()) == 0.0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("sizes", [[1], [3, 0, 5], SIZES, [4096] * 700, [5_000_001]])
def test_gradient_norm_and_clipping(P, dtype, sizes):
    from paper_2209_13258_b200.optim import AdamW
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    ps = make(sizes, dt, 5)
    norm = math.sqrt(sum(float(p.grad.double().square().sum()) for p in ps))
    for max_norm in (norm / 3, norm * 3):
        opt = AdamW(ps, lr=0.0, weight_decay=0.0, max_norm=max_norm)
        opt.step()
        got = opt.grad_norm.tolist()
        # fp32 sums of at most 4096 / 256 * (chunks per block) squares each, then fp64
        assert abs(got[0] - norm) <= 2e-6 * norm
        assert abs(got[1] - min(1.0, max_norm / (norm + 1e-6))) <= 3e-6
        first = opt.grad_norm.clone()
        g = [p.grad.double() * got[1] for p in ps]
        for i, p in enumerate(ps):
            m = states(opt, i)[0]
            assert bool(((m - 0.1 * g[i]).abs() <= 4 * 2.0 ** -24 * g[i].abs() + 1e-37).all())
        opt.step()
        assert torch.equal(opt.grad_norm, first)                     # same gradients, same bits


def test_codes_are_those_of_the_formulas_op_by_op(P):
    """8-bit states: the same codes and scales as the formulas in elementary fp32 operations, bit by bit, over several
    steps (a code that falls on the other side of a tie would move a later scale by some percent)."""
    from paper_2209_13258_b200.optim import AdamW
    n, b1, b2 = 1 << 21, 0.9, 0.95
    rnd = gen(31)
    p = torch.nn.Parameter(rnd(n) * 0.05)
    opt = AdamW([p], lr=1e-3, betas=(b1, b2), state_dtype="e4m3")
    m = v = torch.zeros(n, device="cuda")
    for t in range(4):
        g = rnd(n) * torch.exp(rnd(n // QB, 1)).expand(-1, QB).reshape(-1) * (rnd(n) > -1.5)
        p.grad = g
        opt.step()
        m = m * b1 + g * (1.0 - b1)
        v = v * b2 + (g * g) * (1.0 - b2)
        root = v.sqrt()
        for x, codes, scales in ((m, opt.exp_avg, opt.exp_avg_scale), (root, opt.exp_avg_sq, opt.exp_avg_sq_scale)):
            top = x.view(-1, QB).abs().amax(1)
            c = x.view(-1, QB) * (top.reciprocal() * 448.0)[:, None]
            if x is root:
                c = torch.where(x.view(-1, QB) > 0, c.clamp_min(2.0 ** -9), c)
            want = c.to(torch.float8_e4m3fn).view(-1).float()
            assert torch.equal(codes.float(), want)
            assert torch.equal(scales, top * (1.0 / 448.0))
        m = (opt.exp_avg.float().view(-1, QB) * opt.exp_avg_scale[:, None]).view(-1)
        v = (opt.exp_avg_sq.float().view(-1, QB) * opt.exp_avg_sq_scale[:, None]).view(-1).square()


@pytest.mark.parametrize("scale", [1e-12, 1e12, 1e15])
def test_clipping_of_gradients_far_from_one(P, scale):
    """The coefficient's square is outside fp32's normal range at the largest norm; v is not."""
    from paper_2209_13258_b200.optim import AdamW
    p = torch.nn.Parameter(gen(8)(1 << 20) * 0.05)
    p.grad = gen(9)(1 << 20) * scale
    opt = AdamW([p], lr=1e-3, betas=(0.9, 0.999), max_norm=0.1)
    opt.step()
    coef = float(opt.grad_norm[1])
    m, v = states(opt, 0)
    g = p.grad.double() * coef
    # roundings: of c g, 1 - beta and its product; in v c g twice and its square
    assert bool(((m - 0.1 * g).abs() <= 5 * 2.0 ** -24 * 0.1 * g.abs() + 1e-37).all())
    assert bool(((v - 0.001 * g * g).abs() <= 5 * 2.0 ** -24 * 0.001 * g * g + 1e-37).all())


def test_a_norm_that_is_not_finite_changes_nothing(P):
    from paper_2209_13258_b200.optim import AdamW
    for bad in (float("nan"), float("inf")):
        ps = make(SIZES, torch.bfloat16, 7)
        opt = AdamW(ps, lr=1e-2, master=True, max_norm=1.0, state_dtype="e4m3")
        opt.step()
        keep = [t.clone() for t in (*[p.detach() for p in ps], opt.exp_avg.view(torch.uint8), opt.exp_avg_sq.view(torch.uint8), opt.exp_avg_scale,
                                    opt.exp_avg_sq_scale, opt.master)]
        ps[7].grad[12345] = bad
        opt.step()
        now = (*[p.detach() for p in ps], opt.exp_avg.view(torch.uint8), opt.exp_avg_sq.view(torch.uint8), opt.exp_avg_scale, opt.exp_avg_sq_scale,
               opt.master)
        for a, b in zip(keep, now):
            assert torch.equal(a, b)
        assert not math.isfinite(float(opt.grad_norm[0]))
        ps[7].grad[12345] = 0.0
        opt.step()
        assert math.isfinite(float(opt.grad_norm[0]))
        assert not torch.equal(keep[0], ps[0].detach()) or not torch.equal(keep[-1], opt.master)


def test_zero_gradients_and_tiny_values(P):
    from paper_2209_13258_b200.optim import AdamW
    p = torch.nn.Parameter(torch.ones(600, device="cuda"))
    p.grad = torch.zeros(600, device="cuda")
    opt = AdamW([p], lr=0.1, weight_decay=0.5, state_dtype="e4m3")
    opt.step()
    assert torch.allclose(p.detach(), torch.full_like(p, 0.95), rtol=1e-6)
    assert float(opt.exp_avg_scale.sum()) == 0.0 and float(opt.exp_avg_sq_scale.sum()) == 0.0
    p.grad[:300] = 1e-35                      # below what a block keeps
    p.grad[300:] = torch.linspace(1e-12, 1e-3, 300, device="cuda")
    opt.step()
    assert bool(torch.isfinite(p.detach()).all())
    r = opt.exp_avg_sq.float()
    assert bool((r[512:600] > 0).all())       # a root above zero keeps a code above zero
    assert float(opt.exp_avg_scale[0]) == 0.0


def test_missing_gradients_strides_and_moved_gradients(P):
    from paper_2209_13258_b200.optim import AdamW
    ps = make([512, 300, 1000], torch.float32, 9)
    q = torch.nn.Parameter(torch.zeros(20, 30, device="cuda"))
    q.grad = torch.ones(30, 20, device="cuda").t()                  # not contiguous
    ps[1].grad = None
    old = ps[1].detach().clone()
    opt = AdamW(ps + [q], lr=1e-2, weight_decay=0.0)
    opt.step()
    assert torch.equal(ps[1].detach(), old) and float(opt.exp_avg[512:768].abs().sum()) == 0.0
    assert torch.allclose(q.detach(), torch.full_like(q, -1e-2), rtol=1e-5)
    for p in ps:
        p.grad = torch.full_like(p, 0.5)                            # other addresses than in the step before
    opt.step()
    assert bool((opt.exp_avg[512:812] == 0.5 * (1 - 0.9)).all())


def test_missing_gradients_behind_strided_ones_and_copies(P):
    import copy
    from paper_2209_13258_b200.optim import AdamW
    q = torch.nn.Parameter(torch.zeros(20, 30, device="cuda"))
    q.grad = torch.ones(30, 20, device="cuda").t()
    none, p = torch.nn.Parameter(torch.ones(50, device="cuda")), torch.nn.Parameter(torch.zeros(300, device="cuda"))
    p.grad = torch.full_like(p, -2.0)
    opt = AdamW([q, none, p], lr=1e-2, weight_decay=0.0)
    opt.step()
    assert torch.allclose(q.detach(), torch.full_like(q, -1e-2), rtol=1e-5) and torch.allclose(p.detach(), torch.full_like(p, 1e-2), rtol=1e-5)
    assert bool((none == 1.0).all())
    with pytest.raises(TypeError):      # torch's copy of an optimiser would leave the flat states out
        copy.deepcopy(opt)


def test_state_dict_round_trip(P):
    from paper_2209_13258_b200.optim import AdamW
    a = make(SIZES, torch.bfloat16, 11)
    opt = AdamW(a, lr=1e-2, master=True, state_dtype="e4m3", max_norm=1.0)
    opt.step()
    b = [torch.nn.Parameter(p.detach().clone()) for p in a]
    for p, q in zip(a, b):
        q.grad = p.grad.clone()
    other = AdamW(b, lr=5e-2, master=True, state_dtype="e4m3", max_norm=1.0)
    other.load_state_dict(opt.state_dict())
    opt.step()
    other.step()
    for p, q in zip(a, b):
        assert torch.equal(p, q)
    assert other.steps == 2 and other.param_groups[0]["lr"] == 1e-2
    with pytest.raises(ValueError):
        AdamW(b, state_dtype="fp32").load_state_dict(opt.state_dict())


def test_many_tensors_in_one_call_match_one_by_one(P):
    """More tensors than one launch's table holds."""
    from paper_2209_13258_b200.optim import AdamW
    sizes = [(37 * i) % 900 + 1 for i in range(1500)]
    a = make(sizes, torch.float32, 13)
    b = [torch.nn.Parameter(p.detach().clone()) for p in a]
    for p, q in zip(a, b):
        q.grad = p.grad.clone()
    AdamW(a, lr=1e-2).step()
    for q in b[::97] + b[-1:]:
        AdamW([q], lr=1e-2).step()
    for p, q in list(zip(a, b))[::97] + [(a[-1], b[-1])]:
        assert torch.equal(p, q)


def test_on_another_stream_and_refusals(P):
    from paper_2209_13258_b200.optim import AdamW
    a, b = make([5000], torch.bfloat16, 15), make([5000], torch.bfloat16, 15)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o1, o2 = AdamW(a, max_norm=0.1), AdamW(b, max_norm=0.1)
    s.wait_stream(torch.cuda.current_stream())
    o1.step()
    with torch.cuda.stream(s):
        o2.step()
    torch.cuda.synchronize()
    assert torch.equal(a[0], b[0])
    with pytest.raises(ValueError):
        AdamW(a, state_dtype="int4")
    with pytest.raises(TypeError):
        AdamW([torch.nn.Parameter(torch.zeros(4, device="cuda", dtype=torch.float16))])
    with pytest.raises(TypeError):
        AdamW([a[0], torch.nn.Parameter(torch.zeros(4, device="cuda"))])
    with pytest.raises(RuntimeError):
        AdamW([torch.nn.Parameter(torch.zeros(4))])
    with pytest.raises(RuntimeError):
        o1.add_param_group({"params": b})
