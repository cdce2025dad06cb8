"""The gradient of a sigmoid routing at confident logits, against the formula in 64 bits, relative to its own terms."""
import math

import pytest
import torch

import paper_2209_13258_b200 as P

pytestmark = pytest.mark.gpu
D64 = torch.float64
HALF = 2.0 ** -24


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("low,high", [(-8.0, 8.0), (5.0, 30.0), (12.0, 18.0), (25.0, 80.0), (-80.0, -20.0)])
def test_gradient_keeps_its_digits(low, high, renorm, dtype):
    g = torch.Generator(device="cuda").manual_seed(int(high) + 7)
    T, E, k = 300, 48, 4
    l = (low + (high - low) * torch.rand(T, E, device="cuda", generator=g)).to(dtype)
    idx = torch.rand(T, E, device="cuda", generator=g).argsort(1)[:, :k].to(torch.int32).contiguous()
    dw = torch.randn(T, k, device="cuda", generator=g)
    out = torch.full((T, E), math.nan, device="cuda", dtype=dtype)
    dt = P.DTYPE_FP32 if dtype == torch.float32 else P.DTYPE_BF16
    P.osdp_route_bwd(dw, l, E, dt, idx, T, E, k, P.SCORE_SIGMOID, renorm, 1.5, out, E, check=True)
    mine = l.to(D64).gather(1, idx.long())
    rest = 1.0 / (1.0 + torch.exp(mine))                             # 1 - s
    up = 1.5 * dw.to(D64)
    if renorm:
        r = torch.softmax(torch.nn.functional.logsigmoid(mine), 1)
        # (logsigmoid of a double: -log1p(exp(-l)), good to 2^-52 of itself)
        mean = (up * r).sum(1, keepdim=True)
        d = r * (up - mean) * rest
        size = r * (up.abs() + (up * r).abs().sum(1, keepdim=True)) * rest
    else:
        d = up / (1.0 + torch.exp(-mine)) * rest
        size = d.abs()
    # Half units: s 4 of the exponential, sum, quotient = 6; its sum 6 + 5, the share 6 + 11 + 1 = 18; g 1; the mean 1 + 18 + 1 + 5 = 25,
    # the difference 26; 1 - s 6; their products 26 + 18 + 6 + 2 = 52.
    half = torch.finfo(dtype).eps / 2
    tol = half * d.abs() + 64 * HALF * (1 + half) * size + 2.0 ** -126
    got = out.to(D64).gather(1, idx.long())
    assert bool(((got - d).abs() <= tol).all())
    assert int((out != 0).sum()) <= T * k
