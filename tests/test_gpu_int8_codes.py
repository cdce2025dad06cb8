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


def layer(P, N, K, act, bias=True):
    from paper_2209_13258_b200.nn import Int8Linear, quantize_int8
    g = torch.Generator(device="cuda")
    g.manual_seed(N + K)
    w8, sw = quantize_int8((torch.randn(N, K, device="cuda", generator=g) * 1.5 / K ** 0.5).bfloat16())
    b = torch.randn(N, device="cuda", generator=g) * 0.3 if bias else None
    return Int8Linear(w8, sw, b, act=act), torch.randn(700, K, device="cuda", generator=g).bfloat16()


@pytest.mark.parametrize("N,K", [(1024, 2048), (8200, 1040)])
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("bias", [False, True])
def test_a_token_gives_the_same_bits_whatever_comes_with_it(P, N, K, act, bias):
    """One token, some, and enough for the tile kernel."""
    lin, x = layer(P, N, K, act, bias)
    whole = lin(x)
    for n in (1, 5, 16, 33, 65, 300):
        assert torch.equal(lin(x[:n]), whole[:n]), n


@pytest.mark.parametrize("M", [7, 700])
@pytest.mark.parametrize("act", [1, 2])
def test_activation(P, M, act):
    """Against 64 bits.  The pre-activation has three fp32 roundings (4 * 2^-24 of its terms; GeLU's slope is at most 1.13).
    The activation: the exponent of its power of two carries three roundings of at most 127, its own error and the
    reciprocal's are below 2^-22, which is 2^-15 of the value; the erf form 1 + erf loses up to 2^-22 of |z|.  And half a
    unit in the last place of bf16.  The approximate tanh (2^-11) would be far outside for negative z."""
    from test_gpu_int8 import half_unit, linear64
    from paper_2209_13258_b200.nn import quantize_int8
    lin, x = layer(P, 1024, 2048, act)
    x = x[:M]
    q, s = quantize_int8(x)
    mag, ref = linear64(q, s, lin.weight8, lin.w_scale, lin.bias, act)
    slack = half_unit(ref) + 2.0 ** -20 * mag + 2.0 ** -15 * ref.abs() + 1e-30
    off = (lin(x).double() - ref).abs() - slack
    assert bool((off <= 0).all()), float(off.max())


@pytest.mark.parametrize("M,K", [(1, 16), (1, 512), (8, 752), (1, 768), (1, 784), (9, 128), (16, 368), (16, 384), (16, 400)])
@pytest.mark.parametrize("N", [17760, 17768, 32000, 35536])
def test_few_tokens_of_a_narrow_model_through_a_wide_layer(P, M, K, N):
    """Reductions so short that each warp works by itself, outputs so wide that all sixteen of them have work."""
    from test_gpu_int8 import check, codes, gen, linear64, run
    g = gen(M + K + N)
    x8, w8 = codes(g, M, K), codes(g, N, K)
    sx, sw = torch.rand(M, device="cuda", generator=g) * 0.02 / K ** 0.5, torch.rand(N, device="cuda", generator=g) * 0.02
    bias = torch.randn(N, device="cuda", generator=g)
    out = run(P, x8, sx, w8, sw, bias, 0)
    mag, ref = linear64(x8, sx, w8, sw, bias, 0)
    check(out, mag, ref, 0)


def test_a_graph_of_few_tokens_outlives_calls_with_more(P):
    """Decode graphs beside eager prompts: the graph's codes stay its own, and its replay writes into nobody's memory."""
    lin, x = layer(P, 1024, 2048, 1)
    for n in (4, 40):
        lin, _ = layer(P, 1024, 2048, 1)
        xs = x[:n].clone()
        want = lin(xs)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = lin(xs)
        whole = lin(x)
        mine = [torch.full((n * 2048 // k,), 7, dtype=torch.uint8, device="cuda") for k in (1, 1, 2, 4, 8) for _ in range(8)]
        for _ in range(3):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
        assert all(bool((t == 7).all()) for t in mine)
        assert torch.equal(lin(x), whole)


def test_two_streams_on_one_layer(P):
    lin, x = layer(P, 4096, 2048, 0)
    a, b = x[:4].clone(), x[300:304].clone()
    wants = lin(a), lin(b)
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(200):
        for k, (s, t) in enumerate(zip(streams, (a, b))):
            with torch.cuda.stream(s):
                got[k].append(lin(t))
    torch.cuda.synchronize()
    for k in (0, 1):
        assert all(torch.equal(o, wants[k]) for o in got[k])
