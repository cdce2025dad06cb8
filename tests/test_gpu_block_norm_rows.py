"""The block norm's kernels for many rows (and for rows that need a cluster) on data that is hard on them: means far above
the deviation, a row's variance in one lane's channels, rows that are not finite beside others, r in place of x, absent
parts, an RMS norm beside a layer norm.  Every shape here is beyond what the kernel for few rows takes.  Tolerances as in
test_gpu_block_norm.py.
"""
import pytest

from test_gpu_block_norm import P, backward64, case, check_bwd, forward64, gen, grads_in, half_unit, near, run_bwd, run_fwd  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SHAPES = [(1300, 4096), (20000, 128), (10000, 512), (4900, 264), (4, 16384), (40, 12288)]


def plain(**kw):
    return {"post": 0, "pre": 2, "alpha": 1.0, "beta": 1.0, "eps": 0.0, "w_post": None, "b_post": None, "w_pre": None, "b_pre": None, "gate": None, **kw}


@pytest.mark.parametrize("M,D", SHAPES)
def test_a_mean_far_above_the_deviation(P, M, D):
    rnd = gen(D + M)
    x = rnd(M, D) + 1000.0
    _, u, _ = run_fwd(P, x, None, plain())
    _, uo, _ = forward64(x.double(), None, plain())
    # u's error: the mean's, 2^-24 * 1000 a few times over, against a deviation of 1
    assert bool(((u.double() - uo).abs() <= half_unit(uo) + 5e-4).all())
    # y's norm: values of bf16 about a mean of 64, whose mean is good to a few 2^-24 of it against a deviation of 1; r is p
    y = (rnd(M, D) + 64.0).bfloat16()
    c = plain(post=2, pre=0)
    r, _, _ = run_fwd(P, torch.zeros(M, D, device="cuda"), y, c)
    ro, _, _ = forward64(torch.zeros(M, D, dtype=torch.float64, device="cuda"), y.double(), c)
    assert bool(((r.double() - ro).abs() <= 2e-6 * ro.abs() + 4e-5).all())


@pytest.mark.parametrize("M,D", SHAPES)
@pytest.mark.parametrize("channel", [0, 7, -1])
def test_a_variance_in_one_channel(P, M, D, channel):
    """Nearly all of a row's variance stands in one channel (lane 0's, from whose mean the lanes' means are counted, or the
    last lane's), the others are small numbers on a mean of their own."""
    rnd = gen(D + M + channel)
    x = 0.01 * rnd(M, D) + 0.5
    x[:, channel] = 300.0 + rnd(M)
    y = (0.01 * rnd(M, D) - 0.5).bfloat16()
    y[:, channel] = (-300.0 + rnd(M)).bfloat16()
    for kind in (1, 2):
        c = plain(post=kind, pre=kind, eps=1e-5, beta=0.7)
        r, u, st = run_fwd(P, x, y, c)
        ro, uo, so = forward64(x.double(), y.double(), c)
        near(r, ro, "r")
        near(u, uo, "u")
        scale = torch.stack([y.double().square().mean(1).sqrt(), so[:, 1], ro.square().mean(1).sqrt(), so[:, 3]], 1)
        assert bool(((st.double() - so).abs() <= 2e-6 * scale + 1e-30).all())


@pytest.mark.parametrize("M,D", SHAPES)
@pytest.mark.parametrize("kind", [1, 2])
def test_rows_that_are_not_finite_stay_alone(P, M, D, kind):
    x, y, c, _ = case(P, M, D, kind, kind, torch.bfloat16, seed=4)
    r0, good, _ = run_fwd(P, x, y, c)
    bad = torch.zeros(M, dtype=torch.bool, device="cuda")
    y2, x2 = y.clone(), x.clone()
    for row, what in ((1, float("nan")), (M // 2, float("inf")), (M - 1, float("-inf"))):
        (y2 if row != M // 2 else x2)[row, (row * 8 + 3) % D] = what
        bad[row] = True
    r, u, _ = run_fwd(P, x2, y2, c)
    assert bool(torch.isnan(u[bad].float()).any(1).all())
    assert torch.equal(u[~bad], good[~bad]) and torch.equal(r[~bad], r0[~bad])


@pytest.mark.parametrize("M,D", SHAPES)
@pytest.mark.parametrize("rt", ["bf16", "fp32"])
def test_in_place(P, M, D, rt):
    """r written over x while later rows are still being fetched."""
    for kind in (1, 2):
        x, y, c, _ = case(P, M, D, kind, kind, torch.float32 if rt == "fp32" else torch.bfloat16, seed=9)
        r0, u0, _ = run_fwd(P, x, y, c)
        r1, u1, _ = run_fwd(P, x, y, c, in_place=True)
        assert torch.equal(r0, r1) and torch.equal(u0, u1)


@pytest.mark.parametrize("M,D", SHAPES)
@pytest.mark.parametrize("post,pre,has_y,gate,weights", [(0, 1, True, True, True), (1, 0, True, True, True), (2, 1, True, False, True),
                                                         (1, 2, True, True, False), (0, 0, True, True, True), (0, 2, False, False, True),
                                                         (1, 1, False, True, True), (0, 0, False, False, True)])
def test_parts(P, M, D, post, pre, has_y, gate, weights):
    for rt in (torch.bfloat16, torch.float32):
        x, y, c, wide = case(P, M, D, post, pre, rt, gate=gate, weights=weights, seed=5, alpha=0.9, has_y=has_y)
        y = y if has_y else None
        r, u, st = run_fwd(P, x, y, c)
        ro, uo, so = forward64(x.double(), y.double() if has_y else None, wide)
        near(r, ro, "r")
        if pre:
            near(u, uo, "u")
            assert torch.equal(run_fwd(P, x, y, c, want_r=False, want_stats=False)[1], u)
        absent = [k for k, on in ((0, c["post"]), (1, c["post"]), (2, pre), (3, pre)) if not on]
        assert float(st[:, absent].abs().sum()) == 0.0


@pytest.mark.parametrize("M,D", [(20000, 128), (10000, 512), (4900, 264), (1300, 4096)])
@pytest.mark.parametrize("post,pre", [(1, 1), (2, 2), (2, 1), (1, 2)])
def test_backward(P, M, D, post, pre):
    for rt in (torch.bfloat16, torch.float32):
        x, y, c, wide = case(P, M, D, post, pre, rt, seed=D)
        ro, _, st = forward64(x.double(), y.double(), wide)
        r, st = ro.to(rt), st.float()
        dr, du = grads_in(M, D, rt, M)
        got = run_bwd(P, dr, du, y, r, st, c)
        ref, mag = backward64(dr.double(), du.double(), y.double(), r.double(), st.double(), wide)
        check_bwd(got, ref, mag)


def test_module_gradient_of_a_scaled_stream(P):
    from paper_2209_13258_b200.nn import ResidualNorm
    x, y = (gen(k)(700, 512).bfloat16().requires_grad_(True) for k in (1, 2))
    last = ResidualNorm(512, post="rms", pre=None, gate=False, alpha=0.5)
    r, u = last(x, y)
    assert u is None
    r.sum().backward()
    assert torch.equal(x.grad, torch.full_like(x, 0.5))
