"""Norms, gate and residual sum between two blocks (osdp_block_norm_fwd / _bwd, nn.ResidualNorm) against the formulas
in 64 bits, and the gradients also against differences of the 64-bit forward.

Tolerances.  bf16 outputs: half a unit in the last place plus the fp32 arithmetic before it, whose
error is a few 2^-24 of the row's largest terms: 2e-5 of the row's root mean square covers it.  fp32 outputs of a row:
2e-6 of the value plus 2e-6 of the row's root mean square.  Sums over rows: each term carries the relative error of t
and h (a few 2^-24 of the row's scale) and at most (rows per block + blocks) additions follow one another: 2e-5 of the
sum of magnitudes, a row's t counting with its root mean square added (t is a difference: an element near zero carries
the error of its row).
"""
import pytest

from util import Guarded

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F64 = torch.float64


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


def norm64(v, kind, eps, w, b):
    mean = v.mean(1, keepdim=True) if kind == 2 else torch.zeros(v.shape[0], 1, dtype=F64, device=v.device)
    inv = ((v - mean).square().mean(1, keepdim=True) + eps).rsqrt()
    h = (v - mean) * inv
    out = h * (1.0 if w is None else w)
    return (out if b is None else out + b), h, mean, inv


def forward64(x, y, c):
    """(r, u, stats) of the definition; the tensors and vectors are float64."""
    M = x.shape[0]
    st = torch.zeros(M, 4, dtype=F64, device=x.device)
    r = c["alpha"] * x
    if y is not None:
        p = y
        if c["post"]:
            p, _, st[:, 0:1], st[:, 1:2] = norm64(y, c["post"], c["eps"], c["w_post"], c["b_post"])
        r = r + c["beta"] * (p if c["gate"] is None else p * c["gate"])
    u = None
    if c["pre"]:
        u, _, st[:, 2:3], st[:, 3:4] = norm64(r, c["pre"], c["eps"], c["w_pre"], c["b_pre"])
    return r, u, st


def backward64(dr, du, y, r, st, c):
    """The gradients by the formulas, and the sums of magnitudes of the sums over rows."""
    o, mag = {}, {}
    t = torch.zeros_like(y if y is not None else r) if dr is None else dr
    if c["pre"]:
        h, inv = (r - st[:, 2:3]) * st[:, 3:4], st[:, 3:4]
        a = du if c["w_pre"] is None else du * c["w_pre"]
        d = a - h * (a * h).mean(1, keepdim=True)
        if c["pre"] == 2:
            d = d - a.mean(1, keepdim=True)
            o["db_pre"], mag["db_pre"] = du.sum(0), du.abs().sum(0)
        t = t + d * inv
        o["dw_pre"], mag["dw_pre"] = (du * h).sum(0), (du * h).abs().sum(0)
    o["dx"] = c["alpha"] * t
    if y is not None:
        h, inv = ((y - st[:, 0:1]) * st[:, 1:2], st[:, 1:2]) if c["post"] else (y, torch.ones(y.shape[0], 1, dtype=F64, device=y.device))
        w = 1.0 if c["w_post"] is None else c["w_post"]
        p = h * w + (0.0 if c["b_post"] is None else c["b_post"])
        g = 1.0 if c["gate"] is None else c["gate"]
        bt = c["beta"] * t
        size = bt.abs() + bt.square().mean(1, keepdim=True).sqrt()
        o["dgate"], mag["dgate"] = (bt * p).sum(0), (size * (p.abs() + (h * w).abs())).sum(0)
        if c["post"]:
            o["dw_post"], mag["dw_post"] = (bt * g * h).sum(0), (size * g * h).abs().sum(0)
        if c["post"] == 2:
            o["db_post"], mag["db_post"] = (bt * g).sum(0), (size * g).abs().sum(0)
        q = bt * g * w
        d = q
        if c["post"]:
            d = q - h * (q * h).mean(1, keepdim=True)
        if c["post"] == 2:
            d = d - q.mean(1, keepdim=True)
        o["dy"] = d * inv
    return o, mag


def near(got, ref, what):
    """Elementwise, by the type of `got`, against its row."""
    rms = ref.square().mean(-1, keepdim=True).sqrt()
    slack = half_unit(ref) + 2e-5 * rms if got.dtype == torch.bfloat16 else 2e-6 * ref.abs() + 2e-6 * rms
    off = (got.double() - ref).abs() - (slack + 1e-30)
    assert bool((off <= 0).all()), "%s: %g over the bound" % (what, float(off.max()))


def case(P, M, D, post, pre, rt, gate=True, weights=True, seed=1, alpha=1.0, beta=0.7, has_y=True):
    rnd = gen(seed)
    c = {"post": post if has_y else 0, "pre": pre, "alpha": alpha, "beta": beta, "eps": 1e-5}
    vec = lambda on, at: (at + 0.2 * rnd(D)) if on else None            # noqa: E731
    c["w_post"], c["b_post"] = vec(post and weights and has_y, 1.0), vec(post == 2 and has_y, 0.1)
    c["w_pre"], c["b_pre"] = vec(pre and weights, 1.0), vec(pre == 2, 0.1)
    c["gate"] = vec(gate and has_y, 0.5)
    x = (rnd(M, D) * 1.5 + 0.3 * rnd(D)).to(rt)
    y = (rnd(M, D) * 0.7 + 0.3 * rnd(D) + 0.5).bfloat16() if has_y else None
    wide = {k: (v.double() if torch.is_tensor(v) else v) for k, v in c.items()}
    return x, y, c, wide


def run_fwd(P, x, y, c, int8=False, in_place=False, stream=None, want_r=True, want_stats=True):
    M, D = x.shape
    rt = P.DTYPE_FP32 if x.dtype == torch.float32 else P.DTYPE_BF16
    r = Guarded((M, D), x.dtype)
    u = Guarded((M, D), torch.bfloat16) if c["pre"] and not int8 else None
    if in_place:
        r.t.copy_(x)
        x = r.t
    s = torch.full((M,), float("nan"), device="cuda") if int8 else None
    q = torch.full((M, D), 77, dtype=torch.int8, device="cuda") if int8 else None
    st = Guarded((M, 4), torch.float32)
    P.osdp_block_norm_fwd(x, y, M, D, rt, c["post"], c["w_post"], c["b_post"], c["eps"], c["gate"], c["alpha"], c["beta"], c["pre"],
                          c["w_pre"], c["b_pre"], c["eps"], r.t if want_r else None, q if int8 else (u.t if u else None), s,
                          st.t if want_stats else None, stream=stream, check=True)
    torch.cuda.synchronize()
    for b in (r, u, st):
        if b is not None:
            b.check()
    return r.t, (q, s) if int8 else (u.t if u else None), st.t


SHAPES = [(1, 8), (1, 2048), (3, 64), (5, 264), (130, 520), (1, 8192), (7, 1032), (300, 2048), (1200, 1536), (33, 4608), (200, 8192), (19, 8200),
          (5, 12288), (3, 16384)]


@pytest.mark.parametrize("M,D", SHAPES)
@pytest.mark.parametrize("kind", [1, 2])
@pytest.mark.parametrize("rt", ["bf16", "fp32"])
def test_forward(P, M, D, kind, rt):
    x, y, c, wide = case(P, M, D, kind, kind, torch.float32 if rt == "fp32" else torch.bfloat16, seed=D + M)
    r, u, st = run_fwd(P, x, y, c)
    ro, uo, so = forward64(x.double(), y.double(), wide)
    near(r, ro, "r")
    near(u, uo, "u")
    # the mean is a small number among the row's values: its error is relative to them
    scale = torch.stack([y.double().square().mean(1).sqrt(), so[:, 1], ro.square().mean(1).sqrt(), so[:, 3]], 1)
    assert bool(((st.double() - so).abs() <= 2e-6 * scale + 1e-30).all())


@pytest.mark.parametrize("post,pre,has_y,gate,weights", [(0, 1, True, True, True), (1, 0, True, True, True), (2, 1, True, False, True),
                                                         (1, 2, True, True, False), (0, 0, True, True, True), (0, 2, False, False, True),
                                                         (1, 1, False, True, True), (0, 0, False, False, True)])
def test_forward_parts(P, post, pre, has_y, gate, weights):
    for M, D in ((1, 2048), (67, 1032), (40, 12288)):
        x, y, c, wide = case(P, M, D, post, pre, torch.bfloat16, gate=gate, weights=weights, seed=5, alpha=0.9, has_y=has_y)
        r, u, st = run_fwd(P, x, y, c)
        ro, uo, so = forward64(x.double(), y.double() if has_y else None, wide)
        near(r, ro, "r")
        if pre:
            near(u, uo, "u")
            assert torch.equal(run_fwd(P, x, y, c, want_r=False, want_stats=False)[1], u)
        absent = [k for k, on in ((0, c["post"]), (1, c["post"]), (2, pre), (3, pre)) if not on]
        assert float(st[:, absent].abs().sum()) == 0.0


def test_forward_in_place_and_on_another_stream(P):
    x, y, c, wide = case(P, 257, 2048, 1, 1, torch.float32, seed=9)
    r0, u0, _ = run_fwd(P, x, y, c)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        r1, u1, _ = run_fwd(P, x, y, c, in_place=True)
    assert torch.equal(r0, r1) and torch.equal(u0, u1)


def test_large_mean_and_small_values(P):
    """A mean far above the deviation (its subtraction must not lose it) and rows near the bottom of the range."""
    M, D = 9, 4096
    rnd = gen(3)
    x = (rnd(M, D) + 1000.0).float()
    c = {"post": 0, "pre": 2, "alpha": 1.0, "beta": 1.0, "eps": 0.0, "w_post": None, "b_post": None, "w_pre": None, "b_pre": None, "gate": None}
    _, u, st = run_fwd(P, x, None, c)
    _, uo, so = forward64(x.double(), None, c)
    # u's error: the mean's, 2^-24 * 1000 a few times over, against a deviation of 1
    assert bool(((u.double() - uo).abs() <= half_unit(uo) + 5e-4).all())
    small = (rnd(M, D) * 1e-18).float()
    c["pre"] = 1
    _, u, _ = run_fwd(P, small, None, c)
    near(u, forward64(small.double(), None, c)[1], "u of small rows")
    c["eps"] = 1e-5
    _, u, _ = run_fwd(P, torch.zeros(M, D, device="cuda"), None, c)
    assert float(u.abs().max()) == 0.0


def test_rows_that_are_not_finite_stay_alone(P):
    x, y, c, _ = case(P, 12, 1032, 2, 2, torch.bfloat16, seed=4)
    _, good, _ = run_fwd(P, x, y, c)
    y2 = y.clone()
    y2[3, 17], y2[8, 1] = float("nan"), float("inf")
    _, u, _ = run_fwd(P, x, y2, c)
    bad = torch.zeros(12, dtype=torch.bool, device="cuda")
    bad[3] = bad[8] = True
    assert bool(torch.isnan(u[bad].float()).all()) and torch.equal(u[~bad], good[~bad])


@pytest.mark.parametrize("M,D", [(1, 8), (1, 2048), (5, 264), (70, 1032), (300, 4096), (6, 12288), (3, 16384)])
def test_forward_int8(P, M, D):
    """u as int8: the codes are within rounding of u / scale, the scale is the row's largest magnitude / 127."""
    x, y, c, wide = case(P, M, D, 1, 1, torch.bfloat16, seed=D)
    r, (q, s), _ = run_fwd(P, x, y, c, int8=True)
    ro, uo, _ = forward64(x.double(), y.double(), wide)
    near(r, ro, "r")
    top = uo.abs().amax(1)
    assert bool(((s.double() - top / 127).abs() <= 4e-6 * top / 127).all())
    assert float((q.double() - uo / s.double()[:, None]).abs().max()) <= 0.5 + 127 * 8e-6
    z = torch.zeros_like(x)
    _, (q, s), _ = run_fwd(P, z, torch.zeros_like(y), c, int8=True)
    assert float(s.abs().sum()) == 0.0 and int(q.abs().sum()) == 0


def run_bwd(P, dr, du, y, r, st, c, in_place=False, skip=()):
    ref = r if r is not None else dr
    M, D = ref.shape
    rt = P.DTYPE_FP32 if ref.dtype == torch.float32 else P.DTYPE_BF16
    out = {"dx": Guarded((M, D), ref.dtype)}
    if y is not None:
        out["dy"] = Guarded((M, D), torch.bfloat16)
        out["dgate"] = Guarded((D,), torch.float32)
        if c["post"]:
            out["dw_post"] = Guarded((D,), torch.float32)
        if c["post"] == 2:
            out["db_post"] = Guarded((D,), torch.float32)
    if c["pre"]:
        out["dw_pre"] = Guarded((D,), torch.float32)
    if c["pre"] == 2:
        out["db_pre"] = Guarded((D,), torch.float32)
    for k in skip:
        out.pop(k, None)
    if in_place:
        if dr is not None:
            out["dx"].t.copy_(dr)
            dr = out["dx"].t
        if du is not None and "dy" in out:
            out["dy"].t.copy_(du)
            du = out["dy"].t
    get = lambda k: out[k].t if k in out else None          # noqa: E731
    ws = P.new_workspace(P.osdp_block_norm_workspace_bytes(M, D)[1])
    ws.fill_(255)                                            # nothing in it may matter
    P.osdp_block_norm_bwd(dr, du, y, r, st, M, D, rt, c["post"], c["w_post"], c["b_post"], c["gate"], c["alpha"], c["beta"], c["pre"],
                          c["w_pre"], get("dx"), get("dy"), get("dw_post"), get("db_post"), get("dgate"), get("dw_pre"), get("db_pre"),
                          ws, check=True)
    torch.cuda.synchronize()
    for b in out.values():
        b.check()
    return {k: v.t for k, v in out.items()}


def grads_in(M, D, rt, seed):
    rnd = gen(seed + 77)
    return (rnd(M, D) * 0.1).to(rt), (rnd(M, D) * 0.1).bfloat16()


def check_bwd(got, ref, mag):
    for k, v in got.items():
        if k in ("dx", "dy"):
            near(v, ref[k], k)
        else:
            assert bool(((v.double() - ref[k]).abs() <= 2e-5 * mag[k] + 1e-30).all()), k


@pytest.mark.parametrize("M,D", SHAPES)
@pytest.mark.parametrize("kind", [1, 2])
@pytest.mark.parametrize("rt", ["bf16", "fp32"])
def test_backward(P, M, D, kind, rt):
    rt = torch.float32 if rt == "fp32" else torch.bfloat16
    x, y, c, wide = case(P, M, D, kind, kind, rt, seed=D + M)
    st = forward64(x.double(), y.double(), wide)[2]
    r = forward64(x.double(), y.double(), wide)[0].to(rt)
    st = st.float()
    dr, du = grads_in(M, D, rt, M)
    got = run_bwd(P, dr, du, y, r, st, c)
    ref, mag = backward64(dr.double(), du.double(), y.double(), r.double(), st.double(), wide)
    check_bwd(got, ref, mag)
    again = run_bwd(P, dr, du, y, r, st, c, in_place=True)
    for k in got:
        assert torch.equal(got[k], again[k]), k


@pytest.mark.parametrize("post,pre,has_y,gate,weights,has_dr", [(0, 1, True, True, True, True), (1, 0, True, True, True, True),
                                                                (2, 1, True, False, True, False), (1, 2, True, True, False, True),
                                                                (0, 0, True, True, True, True), (0, 2, False, False, True, True),
                                                                (0, 1, False, False, True, False)])
def test_backward_parts(P, post, pre, has_y, gate, weights, has_dr):
    for M, D in ((1, 2048), (67, 1032), (40, 12288)):
        x, y, c, wide = case(P, M, D, post, pre, torch.bfloat16, gate=gate, weights=weights, seed=5, alpha=0.9, has_y=has_y)
        ro, _, st = forward64(x.double(), y.double() if has_y else None, wide)
        r, st = ro.bfloat16(), st.float()
        dr, du = grads_in(M, D, torch.bfloat16, 3)
        dr, du = dr if has_dr else None, du if pre else None
        got = run_bwd(P, dr, du, y, r if pre else None, st if (pre or c["post"]) else None, c)
        ref, mag = backward64(dr.double() if has_dr else None, du.double() if pre else None, y.double() if has_y else None,
                              r.double(), st.double(), wide)
        check_bwd(got, ref, mag)
        some = run_bwd(P, dr, du, y, r if pre else None, st if (pre or c["post"]) else None, c, skip=("dx", "dw_post", "dw_pre"))
        for k in some:
            assert torch.equal(some[k], got[k]), k


def test_backward_of_no_rows_writes_zero_sums(P):
    D = 2048
    x, y, c, _ = case(P, 0, D, 2, 2, torch.bfloat16, seed=5)
    got = run_bwd(P, x, y, y, x, torch.empty(0, 4, device="cuda"), c)
    for k in ("dgate", "dw_post", "db_post", "dw_pre", "db_pre"):
        assert float(got[k].abs().sum()) == 0.0, k
    run_fwd(P, x, y, c)


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_module_gradients_against_differences(P, kind):
    """loss = sum(r A) + sum(u B) through nn.ResidualNorm; every gradient against the central difference of the 64-bit
    loss along a random direction.  The module's r and u are rounded to bf16 (r: fp32 here), its gradients too, so a
    directional derivative is off by about 2^-8 of the terms' root sum of squares: 1 % of it is allowed."""
    from paper_2209_13258_b200.nn import ResidualNorm
    B_, S, D = 2, 37, 264
    rnd = gen(8)
    m = ResidualNorm(D, post=kind, pre=kind, gate=True, beta=0.6, resid_dtype=torch.float32)
    with torch.no_grad():
        for p in m.parameters():
            p.add_(0.2 * rnd(D))
    x = rnd(B_, S, D).requires_grad_(True)
    y = (rnd(S, B_, D) * 0.5).bfloat16().transpose(0, 1).requires_grad_(True)      # not contiguous
    A, Bm = rnd(B_, S, D) * 0.1, (rnd(B_, S, D) * 0.1).bfloat16()
    r, u = m(x, y)
    assert r.shape == x.shape and r.dtype == torch.float32 and u.dtype == torch.bfloat16
    named = {"x": x, "y": y, **dict(m.named_parameters())}
    grads = dict(zip(named, torch.autograd.grad((r, u), list(named.values()), (A, Bm))))
    k = 2 if kind == "layer" else 1

    def loss(v):
        c = {"post": k, "pre": k, "alpha": m.alpha, "beta": m.beta, "eps": m.eps, "b_post": v.get("b_post"), "b_pre": v.get("b_pre"),
             "w_post": v["w_post"], "w_pre": v["w_pre"], "gate": v["gate"]}
        ro, uo, _ = forward64(v["x"].reshape(-1, D), v["y"].reshape(-1, D), c)
        return float((ro * A.double().view(-1, D)).sum() + (uo * Bm.double().view(-1, D)).sum())

    base = {n: v.detach().double() for n, v in named.items()}
    for n, v in base.items():
        d = rnd(*v.shape).double()
        h = 1e-4
        hi, lo = loss({**base, n: v + h * d}), loss({**base, n: v - h * d})
        want = (hi - lo) / (2 * h)
        got = float((grads[n].double() * d).sum())
        scale = float((grads[n].double() * d).square().sum().sqrt())
        assert abs(got - want) <= 0.01 * scale + 1e-6, (n, got, want, scale)


def test_module_forms(P):
    from paper_2209_13258_b200.nn import ResidualNorm
    rnd = gen(2)
    x, y = rnd(4, 6, 512).bfloat16().requires_grad_(True), rnd(4, 6, 512).bfloat16().requires_grad_(True)
    m = ResidualNorm(512, post="layer", pre="rms")
    r, u = m(x)                                                     # in front of the first block
    assert r is x
    u.sum().backward()
    assert x.grad is not None and m.w_post.grad is None and m.w_pre.grad is not None
    last = ResidualNorm(512, post="rms", pre=None, gate=False, alpha=0.5)
    r, u = last(x, y)
    assert u is None
    r.sum().backward()
    assert torch.equal(x.grad, x.grad) and last.w_post.grad is not None
    r, u = m(x, y)
    g = torch.autograd.grad(r.sum(), [x, y], retain_graph=True)     # u unused: its norm has no gradient
    assert torch.equal(g[0], torch.ones_like(g[0]))
    r8, (q, s) = m.forward_int8(x, y)
    assert torch.equal(r8, r) and q.dtype == torch.int8 and s.shape == (4, 6)
    e = torch.empty(0, 512, dtype=torch.bfloat16, device="cuda")
    r, u = m(e, e)
    assert r.shape == u.shape == (0, 512)
    with pytest.raises(ValueError):
        ResidualNorm(100)
    with pytest.raises(TypeError):
        m(x.float(), y)
    with pytest.raises(ValueError):
        m(x, y[:2])
    with pytest.raises(RuntimeError):
        m(torch.zeros(2, 512, dtype=torch.bfloat16))


def test_captured_in_a_graph(P):
    x, y, c, wide = case(P, 64, 2048, 1, 1, torch.bfloat16, seed=6)
    M, D = x.shape
    r, u, st = torch.empty_like(x), torch.empty_like(y), torch.empty(M, 4, device="cuda")
    dr, du = grads_in(M, D, torch.bfloat16, 3)
    dx, dy, dw = torch.empty_like(x), torch.empty_like(y), torch.empty(D, device="cuda")
    ws = P.new_workspace(P.osdp_block_norm_workspace_bytes(M, D)[1])

    def go():
        P.osdp_block_norm_fwd(x, y, M, D, P.DTYPE_BF16, 1, c["w_post"], None, 1e-5, c["gate"], 1.0, 0.7, 1, c["w_pre"], None, 1e-5, r, u,
                              None, st, check=True)
        P.osdp_block_norm_bwd(dr, du, y, r, st, M, D, P.DTYPE_BF16, 1, c["w_post"], None, c["gate"], 1.0, 0.7, 1, c["w_pre"], dx, dy, dw,
                              None, None, None, None, ws, check=True)

    go()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        go()
    x.copy_(x.roll(1, 0))
    y.copy_(y.roll(1, 0))
    g.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (r, u, dx, dy, dw)]
    go()
    torch.cuda.synchronize()
    for a, b in zip(got, (r, u, dx, dy, dw)):
        assert torch.equal(a, b)
