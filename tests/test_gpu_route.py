"""Routing to experts against its definition in 64 bits: the choice is that of exact arithmetic, ties go to the lower index."""
import math

import pytest
import torch

import paper_2209_13258_b200 as P

pytestmark = pytest.mark.gpu
D64 = torch.float64
HALF = 2.0 ** -24      # of a rounding to fp32
SCORES = {"softmax": P.SCORE_SOFTMAX, "sigmoid": P.SCORE_SIGMOID}


def want(logits, bias, k, score, groups=1, top=1, take=1, renorm=True, scale=1.0):
    """idx, weights in 64 bits."""
    l = logits.to(D64)
    T, E = l.shape
    dead = l == -math.inf
    if score == "softmax":
        s = torch.softmax(l, 1)
        s = torch.where(dead.all(1, keepdim=True), 0.0, s)
    else:
        s = torch.sigmoid(l)
    low = lambda v: torch.where(v.isnan(), -math.inf, v)                       # noqa: E731
    c = low(s + bias.to(D64)) if bias is not None else low(s)
    choice = c if bias is not None else low(l)
    if top < groups:
        per = torch.sort(c.view(T, groups, -1), dim=2, descending=True)[0]
        best = low(per[:, :, :take].sum(2))
        rank = torch.argsort(torch.argsort(best, dim=1, descending=True, stable=True), dim=1)
        out = (rank >= top)[:, :, None].expand(T, groups, E // groups).reshape(T, E)
        # experts that may not be chosen stand behind those that are minus infinity
        first = torch.sort(torch.where(out, -math.inf, choice), dim=1, descending=True, stable=True)[1]
        order = torch.argsort(out.gather(1, first).to(torch.int8), dim=1, stable=True)
        idx = first.gather(1, order)[:, :k]
    else:
        idx = torch.sort(choice, dim=1, descending=True, stable=True)[1][:, :k]
    w = s.gather(1, idx)
    if renorm:
        mine = l.gather(1, idx)
        none = (mine == -math.inf).all(1, keepdim=True)
        # s_j / sum s is the softmax of log s, also where s itself is below the smallest number
        w = torch.where(none, 0.0, torch.softmax(mine if score == "softmax" else torch.nn.functional.logsigmoid(mine), 1))
    return idx, w * scale


def route(logits, bias, k, score, groups=1, top=1, take=1, renorm=True, scale=1.0):
    T, E = logits.shape
    idx = torch.full((T, k), -7, dtype=torch.int32, device="cuda")
    w = torch.full((T, k), math.nan, device="cuda")
    dt = P.DTYPE_FP32 if logits.dtype == torch.float32 else P.DTYPE_BF16
    P.osdp_route_fwd(logits, logits.stride(0) if T else E, dt, bias, T, E, k, SCORES[score], groups, top, take, renorm, scale, idx, w, check=True)
    return idx, w


def check(logits, bias, k, score, spread=64.0, **kw):
    """spread: largest |l - max| that matters."""
    idx, w = route(logits, bias, k, score, **kw)
    i64, w64 = want(logits, bias, k, score, **kw)
    assert torch.equal(idx.long(), i64)
    # exponent's rounding `spread` times 2^-24, exponential 4, sums of up to 37 terms, quotient and scale; a share has them twice
    tol = 2.0 * (spread + 4 + 37 + 3) * HALF
    assert torch.equal(w.isnan(), w64.isnan())
    ok = ~w64.isnan()
    assert bool(((w.to(D64) - w64).abs() <= tol * w64.abs() + 2.0 ** -126)[ok].all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E,k,groups,top,take,bias,renorm", [
    (1, 1, 1, 1, 1, 1, False, True), (1, 64, 2, 1, 1, 1, False, True), (9, 60, 4, 1, 1, 1, False, False), (1777, 60, 4, 4, 2, 2, True, True),
    (300, 256, 8, 8, 4, 2, True, True), (300, 256, 8, 8, 4, 1, False, True), (65, 1000, 16, 1, 1, 1, True, False), (33, 1024, 16, 32, 7, 2, True, True),
    (50, 16, 16, 16, 16, 1, True, True), (50, 16, 3, 16, 3, 2, False, True), (40, 33, 5, 11, 2, 2, True, True), (40, 33, 5, 3, 1, 1, False, False),
    (5000, 8, 2, 1, 1, 1, True, True), (129, 129, 7, 3, 2, 2, True, False)])
def test_choice_and_weights(T, E, k, groups, top, take, bias, renorm, score, dtype):
    g = torch.Generator(device="cuda").manual_seed(T + E + k)
    l = (1.5 * torch.randn(T, E, device="cuda", generator=g)).to(dtype)
    b = 0.1 * torch.randn(E, device="cuda", generator=g) if bias else None
    check(l, b, k, score, groups=groups, top=top, take=take, renorm=renorm, scale=2.5)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,top", [(1, 1), (4, 2)])
def test_equal_scores_go_to_the_lower_index(score, groups, top):
    g = torch.Generator(device="cuda").manual_seed(3)
    l = torch.randint(-2, 3, (500, 64), device="cuda", generator=g).float()
    for bias in (None, torch.zeros(64, device="cuda"), torch.randint(0, 2, (64,), device="cuda", generator=g) * 0.25):
        check(l, bias, 6, score, groups=groups, top=top)
        check(l.bfloat16(), bias, 6, score, groups=groups, top=top)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,top,take", [(1, 1, 1), (8, 3, 2)])
def test_scores_that_fp32_cannot_tell_apart(score, groups, top, take):
    """Biases that level the scores of a row up to their own rounding: what decides is beyond fp32."""
    g = torch.Generator(device="cuda").manual_seed(4)
    row = torch.randn(1, 128, device="cuda", generator=g)
    s = torch.softmax(row.to(D64), 1) if score == "softmax" else torch.sigmoid(row.to(D64))
    bias = (0.75 - s[0]).float()
    l = row.repeat(40, 1)
    l[1::2] += 1e-6 * torch.randn(20, 128, device="cuda", generator=g)
    check(l, bias, 8, score, groups=groups, top=top, take=take)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("E,k,groups,top", [(300, 4, 3, 1), (256, 2, 1, 1), (60, 6, 1, 1), (1024, 16, 8, 2), (64, 8, 4, 3), (512, 1, 1, 1)])
def test_equal_scores_among_near_ones(E, k, groups, top, dtype, score):
    """Few different logits, and biases of some ten neighbouring numbers: an expert's equal may stand beside it and a better
    one behind that."""
    g = torch.Generator(device="cuda").manual_seed(E + k)
    for turn in range(6):
        l = (2.0 * torch.randn(400, E, device="cuda", generator=g)).round().div(2.0).to(dtype)
        for bias in (0.5 - 1e-6 * torch.rand(E, device="cuda", generator=g), 2.0 ** -24 * torch.randint(0, 3, (E,), device="cuda", generator=g), None):
            check(l if bias is not None else l + 2.0 ** -21 * torch.randint(0, 3, l.shape, device="cuda", generator=g).to(dtype), bias, k, score,
                  groups=groups, top=top, take=1 + turn % 2)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,top,take", [(1, 1, 1), (8, 3, 2)])
@pytest.mark.parametrize("mask", [-math.inf, torch.finfo(torch.float32).min, -1e9, 1e9])
def test_experts_masked_by_the_bias(score, groups, top, take, mask):
    g = torch.Generator(device="cuda").manual_seed(11)
    l = torch.randn(300, 64, device="cuda", generator=g)
    bias = 0.1 * torch.randn(64, device="cuda", generator=g)
    for some in (slice(0, 64, 3), slice(5, 64), slice(0, 64), slice(7, 8)):
        b = bias.clone()
        b[some] = mask
        check(l, b, 6, score, groups=groups, top=top, take=take)


@pytest.mark.parametrize("E,k", [(8, 1), (64, 3), (256, 8), (1000, 16)])
def test_scores_of_different_make_at_the_border(E, k):
    """Scores that are nearly all bias beside scores that have none: their roundings differ by far, and a chain of near ties
    may pass from one kind to the other."""
    g = torch.Generator(device="cuda").manual_seed(E + k)
    for turn in range(20):
        l = 3.0 * torch.randn(64, E, device="cuda", generator=g)
        l[:, turn % E] += 9.0                                    # one large share
        s = torch.softmax(l.to(D64), 1)
        bias = (0.5 - s.median(0)[0]).float()
        bias[::2] = (s.max(1)[0].median() - s[:, ::2].median(0)[0]).float()
        # logits such that a row's scores meet: l = log of what is missing to 0.5, one Newton step in 64 bits
        near = (0.6 - bias.to(D64)).clamp_min(1e-9)
        rows = torch.log(near / near.sum()).float().repeat(64, 1)
        rows += 2.0 ** -22 * torch.randn(64, E, device="cuda", generator=g)
        check(rows, bias, k, "softmax")
        check(l, bias, k, "softmax", spread=80.0)
        check(l, bias, k, "sigmoid", spread=80.0)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,k,groups,top", [(32, 2, 1, 1), (64, 16, 4, 3), (128, 8, 1, 1), (1000, 5, 1, 1), (1024, 16, 32, 8)])
def test_masked_experts_among_scores_that_fp32_cannot_tell_apart(score, E, k, groups, top):
    """A masked expert's score is its bias exactly, an expert's beside it the same but for what fp32 cannot hold; more of them
    than a warp has lanes."""
    g = torch.Generator(device="cuda").manual_seed(E)
    row = torch.randn(1, E, device="cuda", generator=g)
    row[0, ::3] = -math.inf
    s = torch.softmax(row.to(D64), 1) if score == "softmax" else torch.sigmoid(row.to(D64))
    bias = (0.75 - s[0]).float()
    bias[::3] = 0.75
    l = row.repeat(16, 1)
    l[1::2] += 1e-7 * torch.randn(8, E, device="cuda", generator=g)
    for take in (1, 2):
        check(l, bias, k, score, groups=groups, top=top, take=take, renorm=False)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("groups,top", [(1, 1), (4, 2)])
@pytest.mark.parametrize("bias", [False, True])
def test_masked_and_broken_logits(score, renorm, groups, top, bias):
    g = torch.Generator(device="cuda").manual_seed(5)
    E, k = 32, 4
    l = torch.randn(12, E, device="cuda", generator=g)
    l[0] = -math.inf                                   # nothing is left
    l[1, 3:] = -math.inf                               # fewer than k are left
    l[2, ::2] = -math.inf
    l[3] = torch.finfo(torch.float32).min              # masked with the lowest value
    l[4, 5:] = torch.finfo(torch.float32).min
    l[5, 7] = math.nan
    l[6] = math.nan
    l[7, 1:31] = math.nan
    l[8] *= 60.0                                       # most scores leave fp32's range
    l[9] = -300.0 + l[9]
    l[10] = torch.finfo(torch.bfloat16).min
    b = 0.1 * torch.randn(E, device="cuda", generator=g) if bias else None
    for rows in (l, l.bfloat16()):
        check(rows, b, k, score, groups=groups, top=top, renorm=renorm, spread=400.0)
    # plus infinity: an index that can be used, whatever the weight
    l[11, 2] = math.inf
    idx, _ = route(l, b, k, score, groups=groups, top=top, renorm=renorm)
    assert bool(((idx >= 0) & (idx < E)).all()) and bool((torch.sort(idx, 1)[0].diff(dim=1) > 0).all())
    assert groups > 1 or int(idx[11, 0]) == 2 or (bias and score == "softmax")


def test_rows_apart_and_unaligned():
    g = torch.Generator(device="cuda").manual_seed(6)
    for dtype in (torch.float32, torch.bfloat16):
        wide = torch.randn(77, 91, device="cuda", generator=g).to(dtype)
        check(wide[:, 7:7 + 60], None, 3, "softmax")
        idx, w = route(wide[:, 7:67], None, 3, "softmax")
        for renorm in (True, False):
            dw = torch.randn(77, 3, device="cuda", generator=g)
            out = torch.full((77, 91), 5.0, device="cuda", dtype=dtype)
            dt = P.DTYPE_FP32 if dtype == torch.float32 else P.DTYPE_BF16
            P.osdp_route_bwd(dw, wide[:, 7:67], 91, dt, idx, 77, 60, 3, P.SCORE_SOFTMAX, renorm, 1.0, out[:, 7:67], 91, check=True)
            assert bool((out[:, :7] == 5.0).all()) and bool((out[:, 67:] == 5.0).all())
            close_gradient(out[:, 7:67], wide[:, 7:67], idx, dw, "softmax", renorm, 1.0)


def gradient(logits, idx, dw, score, renorm, scale):
    """d sum(weights * dw) / d logits in 64 bits by autograd of the definition; an index outside the experts is left out."""
    l = logits.to(D64).requires_grad_()
    E = l.shape[1]
    s = torch.softmax(l, 1) if score == "softmax" else torch.sigmoid(l)
    on = (idx >= 0) & (idx < E)
    w = s.gather(1, idx.long().clamp(0, E - 1)) * on
    if renorm:
        w = w / w.sum(1, keepdim=True).clamp_min(1e-300)
    (scale * w * dw.to(D64) * on).sum().backward()
    return l.grad


def close_gradient(got, logits, idx, dw, score, renorm, scale, spread=32.0):
    d = gradient(logits, idx, dw, score, renorm, scale)
    # a difference of terms as large as scale * sum |dw| times the score: 2 (spread + 40) roundings of each
    size = scale * dw.to(D64).abs().sum(1, keepdim=True).expand_as(d)
    half = torch.finfo(got.dtype).eps / 2
    tol = half * d.abs() + 2 * (spread + 40) * HALF * size + 2.0 ** -126
    assert bool(((got.to(D64) - d).abs() <= tol).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 2), (1777, 60, 4), (300, 256, 8), (65, 1000, 16), (7, 3, 3), (41, 33, 5)])
def test_gradient(T, E, k, score, renorm, dtype):
    g = torch.Generator(device="cuda").manual_seed(T + E)
    l = (1.5 * torch.randn(T, E, device="cuda", generator=g)).to(dtype)
    idx = torch.rand(T, E, device="cuda", generator=g).argsort(1)[:, :k].to(torch.int32).contiguous()
    dw = torch.randn(T, k, device="cuda", generator=g)
    out = torch.full((T, E), math.nan, device="cuda", dtype=dtype)
    dt = P.DTYPE_FP32 if dtype == torch.float32 else P.DTYPE_BF16
    P.osdp_route_bwd(dw, l, E, dt, idx, T, E, k, SCORES[score], renorm, 2.5, out, E, check=True)
    close_gradient(out, l, idx, dw, score, renorm, 2.5)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_gradient_against_differences(score, renorm):
    g = torch.Generator(device="cuda").manual_seed(8)
    T, E, k = 6, 12, 3
    l = torch.randn(T, E, device="cuda", generator=g)
    idx = want(l, None, k, score)[0].to(torch.int32).contiguous()
    dw = torch.randn(T, k, device="cuda", generator=g)
    out = torch.empty_like(l)
    P.osdp_route_bwd(dw, l, E, P.DTYPE_FP32, idx, T, E, k, SCORES[score], renorm, 1.0, out, E, check=True)

    def value(x):
        s = torch.softmax(x, 1) if score == "softmax" else torch.sigmoid(x)
        w = s.gather(1, idx.long())
        return ((w / w.sum(1, keepdim=True) if renorm else w) * dw.to(D64)).sum()
    h = 1e-5
    for t in range(T):
        for e in range(E):
            step = torch.zeros(T, E, dtype=D64, device="cuda")
            step[t, e] = h
            diff = (value(l.to(D64) + step) - value(l.to(D64) - step)) / (2 * h)
            # h^2 times a third derivative, which is below 2 sum |dw|, and the kernel's own roundings
            assert abs(float(diff) - float(out[t, e])) <= float(dw[t].abs().sum()) * (h * h + 150 * HALF) + 1e-9


def test_gradient_of_repeated_and_missing_choices():
    g = torch.Generator(device="cuda").manual_seed(9)
    l = torch.randn(40, 20, device="cuda", generator=g)
    idx = torch.randint(-1, 21, (40, 4), device="cuda", generator=g).to(torch.int32)
    idx[0] = 3
    idx[1] = -1
    idx[2] = 2 ** 31 - 1
    dw = torch.randn(40, 4, device="cuda", generator=g)
    for score in SCORES:
        for renorm in (True, False):
            out = torch.full_like(l, math.nan)
            P.osdp_route_bwd(dw, l, 20, P.DTYPE_FP32, idx, 40, 20, 4, SCORES[score], renorm, 1.0, out, 20, check=True)
            close_gradient(out, l, idx, dw, score, renorm, 1.0)


def test_gradient_where_scores_leave_the_range():
    """The shares of the chosen experts hold where every score of them underflows; masked logits have no gradient."""
    l = torch.tensor([[-200.0, -201.0, -203.0, 0.0], [-1e4, -1e4 - 1, -1e4 - 2, 50.0], [-math.inf, 1.0, 2.0, -math.inf]], device="cuda")
    idx = torch.tensor([[0, 1, 2], [0, 1, 2], [2, 1, 0]], dtype=torch.int32, device="cuda")
    dw = torch.tensor([[1.0, -2.0, 0.5]] * 3, device="cuda")
    r = torch.softmax(l.gather(1, idx.long()).to(D64), 1)
    d = r * (dw - (r * dw).sum(1, keepdim=True))
    for score in SCORES:
        out = torch.empty_like(l)
        P.osdp_route_bwd(dw, l, 4, P.DTYPE_FP32, idx, 3, 4, 3, SCORES[score], True, 1.0, out, 4, check=True)
        # (a sigmoid of -200 is its exponential)
        assert bool(((out.gather(1, idx.long()).to(D64) - d)[:2].abs() <= 1e-5 * dw.abs().sum()).all())
        assert bool((out[:, 3] == 0).all()) and float(out[2, 0]) == 0.0


def test_no_tokens_and_two_streams():
    l = torch.randn(0, 8, device="cuda")
    assert route(l, None, 2, "softmax")[0].shape == (0, 2)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    l = torch.randn(3000, 64, device="cuda")
    torch.cuda.synchronize()
    got = []
    for s in (a, b, a, b):
        with torch.cuda.stream(s):
            got.append(route(l, None, 4, "sigmoid"))
    torch.cuda.synchronize()
    for idx, w in got[1:]:
        assert torch.equal(idx, got[0][0]) and torch.equal(w, got[0][1])
