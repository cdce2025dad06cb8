"""int8 codes are those of their definition in elementary fp32 operations: scale = max / 127 and code = value / scale, both
IEEE divisions, rounded to nearest, ties to even.  No tolerance."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2209_13258_b200 as pkg
    pkg.lib()
    return pkg


@pytest.mark.parametrize("M,K", [(1, 8192), (3, 264), (150, 1032), (4096, 2048)])
def test_codes_and_scales(P, M, K):
    from paper_2209_13258_b200.nn import quantize_int8
    g = torch.Generator(device="cuda")
    g.manual_seed(M + K)
    x = (torch.randn(M, K, device="cuda", generator=g) * torch.exp(3 * torch.randn(M, 1, device="cuda", generator=g))).bfloat16()
    q, s = quantize_int8(x)
    f = x.float()
    # tensor / tensor: torch multiplies by a reciprocal where the divisor is a Python number
    scale = f.abs().amax(1) / torch.full((M,), 127.0, device="cuda")
    assert torch.equal(s, scale)
    want = torch.round(f / scale[:, None])
    off = int((q.float() != want).sum())
    assert off == 0, "%d of %d codes differ" % (off, q.numel())
