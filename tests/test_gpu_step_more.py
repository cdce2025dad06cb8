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


# ---- second moments at the bottom of fp32's range

@pytest.mark.parametrize("state", ["fp32", "e4m3"])
@pytest.mark.parametrize("size", [1e-14, 1e-16, 1e-18, 1e-19, 2e-20])
def test_small_second_moments(P, state, size):
    """eps = 0, so that the update shows the root.  v = 0.001 g^2 has two roundings, in the subnormal range of half of
    2^-149 each: its root is off by a relative 2^-150 / v and the usual 2^-20."""
    from paper_2209_13258_b200.optim import AdamW
    n = 5000
    p = torch.nn.Parameter(torch.zeros(n, device="cuda"))
    p.grad = torch.where(torch.arange(n, device="cuda") % 2 == 0, size, -size) * (1 + gen(3)(n).abs())
    opt = AdamW([p], lr=1.0, betas=(0.9, 0.999), eps=0.0, weight_decay=0.0, state_dtype=state)
    opt.step()
    zero = torch.zeros(n, dtype=F64, device="cuda")
    _, _, v, upd = step64(zero, p.grad.double(), zero, zero, 1, 1.0, 0.9, 0.999, 0.0, 0.0)
    assert bool(((p.detach().double() + upd).abs() <= upd.abs() * (2.0 ** -20 + 2.0 ** -150 / v)).all())
    root = states(opt, 0)[1].sqrt()
    want = v.sqrt()
    off = want * (2.0 ** -22 + 2.0 ** -150 / v)
    if state == "e4m3":
        at = torch.arange(n, device="cuda") // QB
        # (at this beta2 up or down: a whole step of the code)
        off = off + torch.maximum(want * 2.0 ** -3, opt.exp_avg_sq_scale[at].double() * 2.0 ** -9) * 1.0001
    assert bool(((root - want).abs() <= off).all())


def test_codes_of_small_gradients_are_those_of_the_formulas_op_by_op(P):
    """As test_codes_are_those_of_the_formulas_op_by_op, with second moments on both sides of 2^-126 and of 2^-100."""
    from paper_2209_13258_b200.optim import AdamW
    n, b1, b2 = 1 << 20, 0.9, 0.95
    rnd = gen(32)
    p = torch.nn.Parameter(rnd(n) * 0.05)
    opt = AdamW([p], lr=1e-3, betas=(b1, b2), state_dtype="e4m3")
    m = v = torch.zeros(n, device="cuda")
    for t in range(4):
        g = 1e-17 * rnd(n) * torch.exp(2 * rnd(n // QB, 1)).expand(-1, QB).reshape(-1) * (rnd(n) > -1.5)
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


# ---- 8-bit states that have to follow

def dither(n, step, moment):
    """The 20 random bits of every element, by the header's rule."""
    word = 0xFFFFFFFF
    x = torch.arange(n // 8, dtype=torch.int64, device="cuda") ^ ((step * 0xBB67AE85) & word)
    x = ((x ^ (x >> 16)) * 0xB504F333) & word
    x = ((x ^ (x >> 15)) * 0x9E3779B9) & word
    x = ((x ^ (x >> 16)) * 0x9E3779B9) & word
    odd = 2 * (torch.arange(8, device="cuda") + 8 * moment) + 1
    return (((x[:, None] * odd) & word) >> 12).reshape(-1)


def dithered(c, bits):
    a = c.abs()
    up = torch.where(a < 2.0 ** -6, 2.0 ** -6, 0.0)
    a = ((((a + up).view(torch.int32).long() + bits) & 0xFFF00000).int().view(torch.float32) - up).clamp_max(448.0)
    return torch.where(torch.signbit(c), -a, a)


@pytest.mark.parametrize("state,betas", [("e4m3", (0.9, 0.999)), ("e4m3", (0.98, 0.95)), ("e4m3_dithered", (0.9, 0.95)), ("e4m3", (0.975, 0.975))])
def test_dithered_codes_are_those_of_the_formulas_op_by_op(P, state, betas):
    from paper_2209_13258_b200.optim import AdamW
    n, (b1, b2) = 1 << 20, betas
    rnd = gen(33)
    p = torch.nn.Parameter(rnd(n) * 0.05)
    opt = AdamW([p], lr=1e-3, betas=betas, state_dtype=state)
    m = v = torch.zeros(n, device="cuda")
    for t in range(1, 5):
        g = rnd(n) * torch.exp(rnd(n // QB, 1)).expand(-1, QB).reshape(-1) * (rnd(n) > -1.5)
        p.grad = g
        opt.step()
        m = m * b1 + g * (1.0 - b1)
        v = v * b2 + (g * g) * (1.0 - b2)
        for k, (x, codes, scales, beta) in enumerate(((m, opt.exp_avg, opt.exp_avg_scale, b1), (v.sqrt(), opt.exp_avg_sq, opt.exp_avg_sq_scale, b2))):
            top = x.view(-1, QB).abs().amax(1)
            c = (x.view(-1, QB) * (top.reciprocal() * 448.0)[:, None]).view(-1)
            want = dithered(c, dither(n, t, k)) if beta > 0.975 or state == "e4m3_dithered" else c.to(torch.float8_e4m3fn).float()
            if k == 1:
                want = torch.where((x > 0) & (want == 0), 2.0 ** -9, want)
            assert torch.equal(codes.float(), want.to(torch.float8_e4m3fn).float())
            assert torch.equal(scales, top * (1.0 / 448.0))
        m = (opt.exp_avg.float().view(-1, QB) * opt.exp_avg_scale[:, None]).view(-1)
        v = (opt.exp_avg_sq.float().view(-1, QB) * opt.exp_avg_sq_scale[:, None]).view(-1).square()


@pytest.mark.parametrize("noise", [True, False])
@pytest.mark.parametrize("b2,state", [(0.98, "e4m3"), (0.99, "e4m3"), (0.999, "e4m3"), (0.95, "e4m3_dithered")])
def test_second_moments_follow_gradients_that_become_smaller(P, b2, state, noise):
    """Half of every block's gradients become five times smaller; ten half-lives of the second moment later (1 % of the old
    one is left in its root) the stored roots are those of 64 bits.  What the dither adds: about one code's step squared, 1/10
    of the value, to the mean of the square; 6 % in the root is several times that."""
    from paper_2209_13258_b200.optim import AdamW
    n, steps = 32 * QB, int(7 / (1 - b2))
    rnd = gen(34)
    p = torch.nn.Parameter(torch.zeros(n, device="cuda"))
    opt = AdamW([p], lr=0.0, betas=(0.9, b2), weight_decay=0.0, state_dtype=state)
    size = torch.ones(n, device="cuda")
    quiet = torch.arange(n, device="cuda") % 2 == 0
    v = torch.zeros(n, dtype=F64, device="cuda")
    for t in range(2 * steps):
        if t == steps:
            size[quiet] = 0.2
        g = rnd(n)
        p.grad = size * (g if noise else g.sign())
        opt.step()
        v = b2 * v + (1 - b2) * p.grad.double().square()
    root = states(opt, 0)[1].sqrt()
    for part in (quiet, ~quiet):
        ratio = float(root[part].square().mean().sqrt() / v[part].mean().sqrt())
        assert abs(ratio - 1) < 0.06, ratio


# ---- one norm over several optimisers and ranks

def check_clipped(ps, opts, coef):
    """First moments after one step from zero: (1 - beta1) c g."""
    for p, o, i in ((p, o, i) for o in opts for i, p in enumerate(o._params)):
        g = p.grad.double() * coef
        assert bool(((states(o, i)[0] - 0.1 * g).abs() <= 4 * 2.0 ** -24 * g.abs() + 1e-37).all())


@pytest.mark.parametrize("scale", [1 / 3, 3.0])
def test_one_norm_over_two_dtypes(P, scale):
    from paper_2209_13258_b200.optim import AdamW, ClippedStep
    half, full = make([5000, 70001, 8], torch.bfloat16, 3), make([5000, 17, 300], torch.float32, 4)
    for p in full:
        p.grad *= 20
    ps = half + full
    norm = math.sqrt(sum(float(p.grad.double().square().sum()) for p in ps))
    opts = [AdamW(half, lr=1e-3, master=True), AdamW(full, lr=1e-3)]
    both = ClippedStep(opts, max_norm=norm * scale)
    both.step()
    got = both.grad_norm.tolist()
    assert abs(got[0] - norm) <= 2e-6 * norm
    assert abs(got[1] - min(1.0, scale)) <= 3e-6
    check_clipped(ps, opts, got[1])
    assert all(o.steps == 1 for o in opts)
    both.zero_grad()
    assert all(p.grad is None for p in ps)


class Pair:
    """The all-reduce of two ranks that run one after the other: adds what the other one brings."""
    world = 2

    def __init__(self, rank):
        self.rank, self.other = rank, None

    def all_reduce(self, t, tag=None):
        t.add_(self.other)


def two_ranks(step=True):
    from paper_2209_13258_b200.optim import AdamW, ClippedStep
    ranks = []
    for r in (0, 1):
        shard, whole = make([40000, 300], torch.bfloat16, 10 + r), make([5000], torch.bfloat16, 3)
        bias = make([1000], torch.float32, 4)
        for p in shard:
            p.grad *= 1 + 9 * r                       # the ranks' own norms differ by far
        opts = [AdamW([{"params": shard, "sharded": True}, {"params": whole}], lr=1e-2, master=True), AdamW(bias, lr=1e-2)]
        ranks.append((shard, whole + bias, opts, ClippedStep(opts, max_norm=0.5, comm=Pair(r))))
    return ranks


def step_both(ranks):
    sums = [c._local_sums().clone() for *_, c in ranks]
    for r, (*_, c) in enumerate(ranks):
        c.comm.other = sums[1 - r]
        c.step()


def test_one_norm_over_ranks_with_replicated_parameters_beside_shards(P):
    ranks = two_ranks()
    for k in range(3):
        step_both(ranks)
        sharded = sum(float(p.grad.double().square().sum()) for shard, *_ in ranks for p in shard)
        norm = math.sqrt(sharded + sum(float(p.grad.double().square().sum()) for p in ranks[0][1]))
        for shard, rep, opts, c in ranks:
            assert abs(float(c.grad_norm[0]) - norm) <= 2e-6 * norm
            if k == 0:
                check_clipped(shard + rep, opts, float(c.grad_norm[1]))
        assert torch.equal(ranks[0][3].grad_norm, ranks[1][3].grad_norm)
        assert all(torch.equal(p, q) for p, q in zip(ranks[0][1], ranks[1][1]))     # replicated parameters stay the same


def test_a_norm_that_is_not_finite_on_one_rank_changes_nothing_on_any(P):
    ranks = two_ranks()
    step_both(ranks)
    ranks[1][0][0].grad[123] = float("nan")
    before = [p.detach().clone() for shard, rep, *_ in ranks for p in shard + rep]
    step_both(ranks)
    assert all(torch.equal(p, q) for p, q in zip(before, (p for shard, rep, *_ in ranks for p in shard + rep)))
    assert all(math.isnan(float(c.grad_norm[1])) for *_, c in ranks)
