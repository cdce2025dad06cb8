"""Routing where scores reach the end of 64 bits: sigmoids that are 1 and softmax scores that are 0 though their logits differ."""
import math

import pytest
import torch

from test_gpu_route import route, want

pytestmark = pytest.mark.gpu


def order(logits, k):
    return torch.sort(logits.double(), dim=1, descending=True, stable=True)[1][:, :k]


def far_logits(score, T, E, g):
    """Logits whose scores are the same number in 64 bits, but for one expert of the softmax.  Some are equal."""
    if score == "sigmoid":
        return 40.0 + 0.5 * torch.randint(0, 160, (T, E), device="cuda", generator=g).float()
    l = -1000.0 - 8.0 * torch.randint(0, 100, (T, E), device="cuda", generator=g).float()
    l[torch.arange(T, device="cuda"), torch.randint(0, E, (T,), device="cuda", generator=g)] = 0.0
    return l


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,k", [(2, 1), (8, 2), (24, 6), (64, 8), (256, 8), (1024, 16)])
def test_the_larger_logit_wins(score, E, k, dtype):
    g = torch.Generator(device="cuda").manual_seed(E + k)
    l = far_logits(score, 200, E, g).to(dtype)
    for bias in (None, torch.zeros(E, device="cuda"), torch.full((E,), 0.25, device="cuda"), torch.full((E,), -3.0, device="cuda")):
        idx, _ = route(l, bias, k, score)
        assert torch.equal(idx.long(), order(l, k))


def test_two_experts():
    l = torch.tensor([[40.0, 41.0], [41.0, 40.0], [50.0, 50.0]], device="cuda")
    for bias in (None, torch.zeros(2, device="cuda")):
        assert route(l, bias, 1, "sigmoid")[0].flatten().tolist() == [1, 0, 0]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_bias_of_zeros_is_no_bias(score):
    """From ordinary logits to saturated ones, logits a rounding apart among them; with groups too."""
    g = torch.Generator(device="cuda").manual_seed(1)
    for spread in (0.005, 1.0, 30.0, 300.0, 1e4):
        l = spread * torch.randn(400, 64, device="cuda", generator=g)
        l[::2, 32:] = torch.nextafter(l[::2, :32], torch.full_like(l[::2, :32], math.inf))
        for groups, top, take in ((1, 1, 1), (8, 3, 1), (8, 3, 2)):
            plain = route(l, None, 6, score, groups=groups, top=top, take=take)
            zeros = route(l, torch.zeros(64, device="cuda"), 6, score, groups=groups, top=top, take=take)
            assert torch.equal(plain[0], zeros[0]) and torch.equal(plain[1], zeros[1])
            if groups == 1:
                assert torch.equal(plain[0].long(), order(l, 6))


@pytest.mark.parametrize("mask", [-math.inf, torch.finfo(torch.float32).min, -1e30])
def test_behind_a_mask_all_are_equal(mask):
    """A mask leaves nothing of the score: lowest index first, also where the logits would tell them apart."""
    g = torch.Generator(device="cuda").manual_seed(2)
    l = far_logits("sigmoid", 100, 40, g)
    bias = torch.full((40,), mask, device="cuda")
    free = [7, 19, 33]
    bias[free] = 0.0
    idx, _ = route(l, bias, 8, "sigmoid")
    here = torch.tensor(free, device="cuda")
    assert torch.equal(idx[:, :3].long(), here[order(l[:, free], 3)])
    assert bool((idx[:, 3:].long() == torch.tensor([0, 1, 2, 3, 4], device="cuda")).all())


def test_different_biases_decide_before_the_logits():
    g = torch.Generator(device="cuda").manual_seed(3)
    l = far_logits("sigmoid", 100, 32, g)
    bias = torch.randperm(32, device="cuda", generator=g).float() * 2.0 ** -22
    idx, _ = route(l, bias, 5, "sigmoid")
    assert bool((idx.long() == torch.argsort(bias, descending=True)[:5]).all())
    assert torch.equal(idx.long(), want(l, bias, 5, "sigmoid")[0])
