"""The activation of the experts' products where its output is small, and a token alone beside the same one among others.

Rows, weights and biases are small multiples of powers of two, so that every sum is exact and only the activation and the
rounding of its output are left."""
import math

import pytest
import torch

import paper_2209_13258_b200 as P
from test_gpu_experts import BF16, D64, HALF16, make_plan, rows_of

pytestmark = pytest.mark.gpu


def gelu(z, act):
    """Without a difference, so that a small output has all its digits in 64 bits too."""
    if act == P.ACT_GELU_ERF:
        return 0.5 * z * torch.erfc(-z * math.sqrt(0.5))
    return z / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))


def problem(T, E, k, N, K, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    whole = lambda top, *n: torch.randint(-top, top + 1, n, device="cuda", generator=g).float()      # noqa: E731
    x, w, bias = whole(4, T, K) / 4, whole(8, E, N, K) / 16, whole(96, E, N) / 16
    idx = torch.rand(T, E, device="cuda", generator=g).argsort(1)[:, :k].to(torch.int32).contiguous()
    return x.to(BF16), w.to(BF16), bias, idx


def product(x, w, bias, idx, act):
    """out and z as [T, k, N]."""
    T, k = idx.shape
    E, N, K = w.shape
    plan, pos, R = make_plan(idx, E)
    rows = rows_of(x[:, None].expand(T, k, K), pos, R)
    out, z = (torch.empty(R, N, dtype=BF16, device="cuda") for _ in range(2))
    ws = P.new_workspace(256)
    P.osdp_expert_linear_fwd(rows, plan, w, 0, bias, T, k, E, N, K, act, out, z, ws, check=True)
    return out[pos.long()], z[pos.long()]


@pytest.mark.parametrize("act", [P.ACT_GELU_TANH, P.ACT_GELU_ERF])
@pytest.mark.parametrize("T,E,k,N,K", [(300, 4, 2, 264, 16), (2000, 3, 2, 1024, 32), (8, 4, 2, 264, 16), (40, 8, 1, 520, 32), (1, 2, 2, 72, 8)])
def test_small_outputs_keep_their_digits(T, E, k, N, K, act):
    x, w, bias, idx = problem(T, E, k, N, K)
    out, z = product(x, w, bias, idx, act)
    i = idx.long()
    want = torch.einsum("tk,tjnk->tjn", x.to(D64), w.to(D64)[i]) + bias.to(D64)[i]
    assert torch.equal(z, want.to(BF16)) and float(want.min()) < -5.0 and float(want.max()) > 5.0
    # tanh form: the exponent 2 u has three roundings, 3 |2 u| 2^-24 of h = 1 / (1 + e^2u); exponential 2^-22, sum, reciprocal 2^-22,
    # product.  erf form: z^2 times the argument's two roundings, the function's units, two products.  Both below 2^-14 for |z| < 16.
    # (A share h below fp32's smallest normal number counts as zero: |z| 2^-126.)
    a = gelu(want, act)
    assert float(want.abs().max()) < 16.0
    assert bool(((out.to(D64) - a).abs() <= (2.0 ** -14 + HALF16 * (1 + 2.0 ** -14)) * a.abs() + 2.0 ** -122).all())


@pytest.mark.parametrize("act", [P.ACT_GELU_TANH, P.ACT_GELU_ERF])
def test_a_token_alone_has_the_outputs_that_it_has_in_a_batch(act):
    x, w, bias, idx = problem(2000, 4, 2, 520, 32, seed=1)
    all_of_them = product(x, w, bias, idx, act)
    for n in (1, 8, 9, 300):
        for a, b in zip(product(x[:n], w, bias, idx[:n].contiguous(), act), all_of_them):
            assert torch.equal(a, b[:n])
