"""int8 linear layer (osdp_quantize_rows_i8, osdp_split_linear_fwd_i8, nn.Int8Linear) against 64 bits.

The integer sums are exact, so against the definition on the same codes only the epilogue's roundings remain: four fp32
roundings (2^-20 of the magnitudes) and half a unit in the last place of the bf16 output.  The activation of many tokens uses the framework's
approximate tanh: 2^-11 of it, times |z| / 2.
"""
import math

import pytest

from util import Guarded

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


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
    return g


def half_unit(v):
    """Half a unit in the last place of bf16 (8 significant bits) at |v|: what rounding to nearest may cost."""
    return torch.ldexp(torch.ones_like(v), torch.frexp(v.abs().clamp_min(1e-300))[1] - 9)


def codes(g, *n):
    return torch.randint(-127, 128, n, device="cuda", generator=g, dtype=torch.int8)


def linear64(x8, sx, w8, sw, bias, act):
    """Magnitude of what is added up to the pre-activation, and the output."""
    z = (x8.double() @ w8.double().t()) * sx.double()[:, None] * sw.double()
    mag = z.abs()
    if bias is not None:
        z, mag = z + bias.double(), mag + bias.double().abs()
    if act == 1:
        return mag, 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == 2:
        return mag, 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    return mag, z


def run(P, x8, sx, w8, sw, bias, act, k=1, split=0, offset=0):
    M, K = x8.shape
    N = w8.shape[0]
    flat = torch.cat([torch.full((offset,), 99, dtype=torch.int8, device="cuda"), w8.reshape(-1)])
    out = Guarded((M, N), torch.bfloat16)
    ws = P.new_workspace(P.osdp_split_linear_workspace_bytes(max(M, 1), N, K, k, split, act, P.OP_LINEAR_FWD)[1])
    P.osdp_split_linear_fwd_i8(x8, sx, flat, offset, sw, bias, M, N, K, k, split, act, out.t, ws, check=True)
    torch.cuda.synchronize()
    out.check()
    rc, st = P.osdp_read_device_status(ws)
    assert rc == 0 and st == 0
    return out.t


def check(out, mag, ref, act):
    slack = half_unit(ref) + 2.0 ** -20 * mag + 1e-30
    if act == 1:
        slack = slack + 2.0 ** -11 * mag
    if act == 2:
        slack = slack + 1e-6 * mag
    off = (out.double() - ref).abs() - slack
    assert bool((off <= 0).all()), float(off.max())


@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 16, 17, 31, 32, 33, 63, 128, 129, 300, 1000])
@pytest.mark.parametrize("N,K", [(8, 16), (72, 80), (520, 1040), (2056, 2064)])
def test_product(P, M, N, K):
    g = gen(M * 7 + N)
    x8, w8 = codes(g, M, K), codes(g, N, K)
    sx, sw = torch.rand(M, device="cuda", generator=g) * 0.02 / math.sqrt(K), torch.rand(N, device="cuda", generator=g) * 0.02
    act = (M + N // 8) % 3
    bias = torch.randn(N, device="cuda", generator=g) if M % 2 else None
    out = run(P, x8, sx, w8, sw, bias, act, offset=32 if M % 3 == 0 else 0)
    mag, ref = linear64(x8, sx, w8, sw, bias, act)
    check(out, mag, ref, act)


@pytest.mark.parametrize("M,N,K", [(4096, 4096, 512), (16384, 1024, 256), (2000, 8192, 1024), (3000, 6160, 2064), (260, 16384, 4096)])
def test_wide_tiles(P, M, N, K):
    """Every tile shape of the tile kernel: CTA pairs on 256- and 512-wide tiles, ragged edges."""
    g = gen(N + K)
    x8, w8 = codes(g, M, K), codes(g, N, K)
    sx, sw = torch.rand(M, device="cuda", generator=g) * 0.001, torch.rand(N, device="cuda", generator=g) * 0.02
    bias = torch.randn(N, device="cuda", generator=g)
    for act in (0, 1):
        out = run(P, x8, sx, w8, sw, bias, act)
        for lo in range(0, M, 2048):
            mag, ref = linear64(x8[lo:lo + 2048], sx[lo:lo + 2048], w8, sw, bias, act)
            check(out[lo:lo + 2048], mag, ref, act)


@pytest.mark.parametrize("M,N,K", [(1, 520, 8192), (1, 64, 32), (2, 2056, 8192), (3, 520, 1040), (4, 4096, 4096), (4, 264, 8192), (7, 520, 1040),
                                   (40, 520, 1040), (300, 1024, 1040), (1, 8200, 16384), (1, 72, 16400)])
def test_bf16_tokens_give_the_same_bits_as_quantised_ones(P, M, N, K):
    """x_scale NULL: whichever kernel quantises, the codes are those of the quantiser."""
    g = gen(M + K)
    x = (torch.randn(M, K, device="cuda", generator=g) * 3).bfloat16()
    w8, sw = codes(g, N, K), torch.rand(N, device="cuda", generator=g) * 0.01
    bias = torch.randn(N, device="cuda", generator=g)
    q, s = torch.empty(M, K, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    P.osdp_quantize_rows_i8(x, M, K, q, s, check=True)
    want = run(P, q, s, w8, sw, bias, 1)
    ws = P.new_workspace(P.osdp_i8_workspace_bytes(M, K)[1])
    out = Guarded((M, N), torch.bfloat16)
    P.osdp_split_linear_fwd_i8(x, None, w8, 0, sw, bias, M, N, K, 1, 0, 1, out.t, ws, check=True)
    torch.cuda.synchronize()
    out.check()
    assert torch.equal(out.t, want)
    assert P.osdp_split_linear_fwd_i8(x, None, w8, 0, sw, bias, M, N, K, 1, 0, 1, out.t, P.new_workspace(256)) == 5


@pytest.mark.parametrize("M,N,K", [(5, 1024, 1024), (300, 1024, 1024), (4096, 2048, 2048)])
@pytest.mark.parametrize("split", [0, 1])
def test_slices_give_the_same_bits(P, M, N, K, split):
    g = gen(3)
    x8, w8 = codes(g, M, K), codes(g, N, K)
    sx, sw = torch.rand(M, device="cuda", generator=g), torch.rand(N, device="cuda", generator=g)
    whole = run(P, x8, sx, w8, sw, None, 0)
    for k in (2, 4, 7):
        L = -(-(N if split == 0 else K) // k)
        if (-(-L // 8) * 8) % 16:
            assert P.osdp_split_linear_fwd_i8(x8, sx, w8, 0, sw, None, M, N, K, k, split, 0, whole, P.new_workspace(256)) == 4
            continue
        assert torch.equal(run(P, x8, sx, w8, sw, None, 0, k=k, split=split), whole)


@pytest.mark.parametrize("M", [3, 64])
def test_extreme_codes_do_not_overflow(P, M):
    K, N = 131056, 16
    x8 = torch.full((M, K), -128, dtype=torch.int8, device="cuda")
    w8 = torch.full((N, K), -128, dtype=torch.int8, device="cuda")
    w8[1::2] = 127
    one = torch.ones(M, device="cuda")
    sw = torch.full((N,), 2.0 ** -20, device="cuda")
    out = run(P, x8, one, w8, sw, None, 0)
    mag, ref = linear64(x8, one, w8, sw, None, 0)
    check(out, mag, ref, 0)


@pytest.mark.parametrize("M,K", [(1, 8), (1, 8192), (5, 264), (150, 1032), (400, 2048), (149, 16384), (3, 131064)])
def test_quantiser(P, M, K):
    g = gen(K + M)
    x = (torch.randn(M, K, device="cuda", generator=g) * torch.exp(torch.randn(M, 1, device="cuda", generator=g))).bfloat16()
    if M > 3:
        x[1] = 0
        x[2] *= 1e-36
    q = torch.full((M + 2, K), 55, dtype=torch.int8, device="cuda")
    s = torch.full((M + 2,), 55.0, device="cuda")
    P.osdp_quantize_rows_i8(x, M, K, q, s, check=True)
    torch.cuda.synchronize()
    assert bool((q[M:] == 55).all()) and bool((s[M:] == 55).all())
    top = x.double().abs().amax(1)
    live = top >= 2.0 ** -100
    want = torch.where(live, top / 127, 0.0)
    assert bool(((s[:M].double() - want).abs() <= 2.0 ** -23 * want).all())
    ratio = torch.where(live[:, None], x.double() / want.clamp_min(1e-300)[:, None], 0.0)
    assert float((q[:M].double() - ratio).abs().max()) <= 0.5 + 127 * 2.0 ** -22
    assert int(q[:M].abs().max()) <= 127


def test_rows_that_are_not_finite(P):
    """An infinity or a NaN in a token makes that token's outputs NaN and no other's."""
    from paper_2209_13258_b200.nn import Int8Linear, quantize_int8
    for M in (12, 200):
        g = gen(4)
        x = torch.randn(M, 512, device="cuda", generator=g).bfloat16()
        w8, sw = quantize_int8(torch.randn(264, 512, device="cuda", generator=g).bfloat16())
        layer = Int8Linear(w8, sw)
        good = layer(x)
        x[3, 100], x[7, 0] = float("inf"), float("nan")
        out = layer(x)
        bad = torch.zeros(M, dtype=torch.bool, device="cuda")
        bad[3] = bad[7] = True
        assert bool(torch.isnan(out[bad].float()).all()) and torch.equal(out[~bad], good[~bad])


def test_module(P):
    from paper_2209_13258_b200.nn import Int8Linear, ResidualNorm, SplitLinear, quantize_int8
    lin = SplitLinear(512, 1040, act=P.ACT_GELU_TANH)
    with torch.no_grad():
        lin.bias.normal_(0, 0.1)
    q = Int8Linear.from_linear(lin)
    g = gen(5)
    x = torch.randn(2, 70, 512, device="cuda", generator=g).bfloat16()
    y, y8 = lin(x).detach().double(), q(x).double()
    # quantisation noise: two roundings to 1/127 of the largest of 512 normal values (about 3.3 deviations)
    assert float((y - y8).norm() / y.norm()) < 0.02
    pair = quantize_int8(x)
    assert torch.equal(q(pair).double(), y8) and pair[1].shape == (2, 70)
    xt = x.transpose(0, 1)
    assert torch.equal(q(xt), q(xt.contiguous()))
    assert q(x[:0]).shape == (0, 70, 1040)
    norm = ResidualNorm(512)
    _, u8 = norm.forward_int8(x, x)
    assert q(u8).shape == (2, 70, 1040)
    with pytest.raises(TypeError):
        q(x.float())
    with pytest.raises(ValueError):
        Int8Linear(torch.zeros(8, 24, dtype=torch.int8, device="cuda"), torch.ones(8, device="cuda"))
    with pytest.raises(ValueError):
        Int8Linear(torch.zeros(8, 32, dtype=torch.int8, device="cuda"), torch.ones(9, device="cuda"))


def test_on_another_stream_and_in_a_graph(P):
    from paper_2209_13258_b200.nn import Int8Linear, quantize_int8
    g = gen(6)
    w8, sw = quantize_int8(torch.randn(1024, 512, device="cuda", generator=g).bfloat16())
    layer = Int8Linear(w8, sw)
    for M in (4, 256):
        x = torch.randn(M, 512, device="cuda", generator=g).bfloat16()
        want = layer(x)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got = layer(x)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = layer(x)
        x.neg_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, layer(x))
