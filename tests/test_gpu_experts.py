"""The experts' rows and products against plain forms in 64 bits."""
import math

import pytest
import torch

import paper_2209_13258_b200 as P

pytestmark = pytest.mark.gpu
D64, BF16 = torch.float64, torch.bfloat16
HALF16, HALF32 = 2.0 ** -8, 2.0 ** -24
MARK = 77.0            # what rows that must not be touched hold


def layout(idx, E):
    """offsets [E + 1], counts [E], pos like idx (-1: none)."""
    flat = idx.reshape(-1).long()
    on = (flat >= 0) & (flat < E)
    counts = torch.bincount(flat[on], minlength=E)
    padded = (counts + 63) // 64 * 64
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=idx.device), padded.cumsum(0)])
    pos = torch.full_like(flat, -1)
    for e in range(E):
        mine = (flat == e).nonzero().view(-1)
        pos[mine] = offsets[e] + torch.arange(len(mine), device=idx.device)
    return offsets, counts, pos.view(idx.shape)


def make_plan(idx, E):
    T, k = idx.shape
    rc, R, ints = P.osdp_expert_rows(T, k, E)
    assert rc == 0
    plan = torch.full((ints,), -9, dtype=torch.int32, device="cuda")
    pos = torch.full((T, k), -9, dtype=torch.int32, device="cuda")
    P.osdp_expert_plan(idx, T, k, E, plan, pos, check=True)
    return plan, pos, R


def choices(T, k, E, how, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + T + E)
    if how == "one":
        return torch.full((T, k), E - 1, dtype=torch.int32, device="cuda")
    if how == "holes":
        return torch.randint(-1, E + 1, (T, k), device="cuda", generator=g).to(torch.int32)
    weight = torch.rand(E, device="cuda", generator=g) ** (3 if how == "skewed" else 0)
    if k <= E:
        return torch.multinomial(weight.expand(max(T, 1), E) + 1e-9, k, generator=g)[:T].to(torch.int32).contiguous()
    return torch.randint(0, E, (T, k), device="cuda", generator=g).to(torch.int32)


SHAPES = [(1, 2, 8, "even"), (37, 2, 16, "skewed"), (300, 3, 5, "holes"), (1777, 4, 60, "skewed"), (64, 1, 1, "one"), (513, 2, 4, "one"),
          (100, 1, 1024, "even"), (20000, 8, 256, "skewed"), (9000, 2, 3, "holes")]


@pytest.mark.parametrize("T,k,E,how", SHAPES)
def test_plan(T, k, E, how):
    idx = choices(T, k, E, how)
    plan, pos, R = make_plan(idx, E)
    offsets, counts, want = layout(idx, E)
    assert torch.equal(plan[:E + 1].long(), offsets) and torch.equal(plan[E + 1:2 * E + 1].long(), counts)
    assert torch.equal(pos.long(), want)
    assert int(offsets[E]) <= R
    for tile, at in ((128, 2 * E + 1), (256, 3 * E + 2)):
        tiles = (counts + tile - 1) // tile
        assert torch.equal(plan[at:at + E + 1].long(), torch.cat([tiles[:0].new_zeros(1), tiles.cumsum(0)]))
    live = counts.nonzero().view(-1)
    assert int(plan[5 * E + 3]) == len(live) and torch.equal(plan[4 * E + 3:4 * E + 3 + len(live)].long(), live)


def test_plan_of_nothing_and_of_no_choice():
    plan, pos, R = make_plan(torch.empty(0, 2, dtype=torch.int32, device="cuda"), 6)
    assert R == 0 and bool((plan[:13] == 0).all())
    plan, pos, R = make_plan(torch.tensor([[-1, 6], [2 ** 31 - 1, -2 ** 31]], dtype=torch.int32, device="cuda"), 6)
    assert bool((plan[:13] == 0).all()) and bool((pos == -1).all())


def rows_of(values, pos, R, fill=0.0):
    """values [T, k, D] in their rows."""
    rows = torch.full((R, values.shape[2]), fill, dtype=values.dtype, device="cuda")
    on = pos >= 0
    rows[pos[on].long()] = values[on]
    return rows


def used(plan, E):
    return int(plan[E])


@pytest.mark.parametrize("D", [8, 1032, 8192])
@pytest.mark.parametrize("T,k,E,how", SHAPES[:6])
def test_dispatch_and_combine(T, k, E, how, D):
    g = torch.Generator(device="cuda").manual_seed(D + T)
    idx = choices(T, k, E, how)
    plan, pos, R = make_plan(idx, E)
    end = used(plan, E)
    x = torch.randn(T, D, device="cuda", generator=g).to(BF16)
    w = torch.randn(T, k, device="cuda", generator=g)
    got = torch.full((R, D), MARK, dtype=BF16, device="cuda")
    P.osdp_expert_dispatch(x, plan, pos, None, None, T, k, E, D, got, None, check=True)
    assert torch.equal(got[:end], rows_of(x[:, None].expand(T, k, D), pos, R)[:end])
    assert bool((got[end:] == MARK).all())
    got.fill_(MARK)
    P.osdp_expert_dispatch(x, plan, pos, w, None, T, k, E, D, got, None, check=True)
    scaled = (x.float()[:, None] * w[:, :, None]).to(BF16)          # one rounding to fp32, one to bf16, in the kernel as here
    assert torch.equal(got[:end], rows_of(scaled, pos, R)[:end]) and bool((got[end:] == MARK).all())
    y = torch.randn(T, k, D, device="cuda", generator=g).to(BF16)
    rows = rows_of(y, pos, R, fill=math.nan)                         # whatever lies between the experts is not read
    on = (pos >= 0).to(D64)
    for weights in (w, None):
        out = torch.full((T, D), math.nan, dtype=BF16, device="cuda")
        P.osdp_expert_combine(rows, plan, pos, weights, T, k, E, D, out, check=True)
        ww = (w.to(D64) if weights is not None else torch.ones_like(w, dtype=D64)) * on
        want = (y.to(D64) * ww[:, :, None]).sum(1)
        size = (y.to(D64).abs() * ww.abs()[:, :, None]).sum(1)
        assert bool(((out.to(D64) - want).abs() <= HALF16 * want.abs() + k * HALF32 * (1 + HALF16) * size).all())
    # backward of combine: rows as the weighted dispatch, and the dot products
    got.fill_(MARK)
    dw = torch.full((T, k), math.nan, device="cuda")
    P.osdp_expert_dispatch(x, plan, pos, w, rows, T, k, E, D, got, dw, check=True)
    assert torch.equal(got[:end], rows_of(scaled, pos, R)[:end]) and bool((got[end:] == MARK).all())
    want = (x.to(D64)[:, None] * y.to(D64)).sum(2) * on
    size = (x.to(D64).abs()[:, None] * y.to(D64).abs()).sum(2) * on
    assert bool(((dw.to(D64) - want).abs() <= (D / 32 + 16) * HALF32 * size).all())


def test_no_tokens():
    T, k, E = 0, 2, 4
    plan, pos, R = make_plan(torch.empty(0, 2, dtype=torch.int32, device="cuda"), E)
    none = torch.empty(0, 64, dtype=BF16, device="cuda")
    P.osdp_expert_dispatch(none, plan, pos, None, None, T, k, E, 64, none, None, check=True)
    P.osdp_expert_combine(none, plan, pos, None, T, k, E, 64, none, check=True)
    w, db = torch.randn(E, 64, 64, device="cuda").to(BF16), torch.ones(E, 64, device="cuda")
    dw = torch.ones(E, 64, 64, device="cuda")
    ws = P.new_workspace(P.osdp_expert_linear_workspace_bytes(T, k, E, 64, 64, 0, P.OP_LINEAR_BWD)[1])
    P.osdp_expert_linear_fwd(none, plan, w, 0, None, T, k, E, 64, 64, 0, none, None, ws, check=True)
    P.osdp_expert_linear_bwd(none, none, plan, w, 0, None, T, k, E, 64, 64, 0, none, dw, 0, P.DTYPE_FP32, P.FLAG_ACCUMULATE_DW, None, ws, check=True)
    assert bool((dw == 1).all())
    P.osdp_expert_linear_bwd(none, none, plan, w, 0, None, T, k, E, 64, 64, 0, none, dw, 0, P.DTYPE_FP32, 0, db, ws, check=True)
    assert bool((dw == 0).all()) and bool((db == 0).all())


def gelu(z, act):
    if act == P.ACT_GELU_TANH:
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    return 0.5 * z * torch.erfc(-z * math.sqrt(0.5)) if act == P.ACT_GELU_ERF else z


def gelu_grad(z, act):
    z = z.detach().clone().requires_grad_()
    gelu(z, act).sum().backward()
    return z.grad


class Problem:
    """Rows, weights and gradients of one set of choices; rows behind the last expert's hold NaN."""

    def __init__(self, T, k, E, how, N, K, bias=True, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed + N + K)
        self.T, self.k, self.E, self.N, self.K = T, k, E, N, K
        self.idx = choices(T, k, E, how)
        self.plan, self.pos, self.R = make_plan(self.idx, E)
        self.end = used(self.plan, E)
        rnd = lambda *n: torch.randn(*n, device="cuda", generator=g)                # noqa: E731
        self.x, self.dy, self.z = (self._rows(rnd(T, k, n).to(BF16)) for n in (K, N, N))
        self.flat = (rnd(E * N * K + 64) * K ** -0.5).to(BF16)
        self.w = self.flat[64:].view(E, N, K)
        self.bias = 0.3 * rnd(E, N) if bias else None
        self.offsets, self.counts = self.plan[:E + 1].tolist(), self.plan[E + 1:2 * E + 1].tolist()

    def _rows(self, v):
        r = rows_of(v, self.pos, self.R)
        r[self.end:] = math.nan
        return r

    def ws(self, act, op):
        return P.new_workspace(P.osdp_expert_linear_workspace_bytes(self.T, self.k, self.E, self.N, self.K, act, op)[1])

    def experts(self):
        for e in range(self.E):
            if self.counts[e]:
                yield e, slice(self.offsets[e], self.offsets[e] + self.counts[e])

    def between(self):
        keep = torch.ones(self.R, dtype=torch.bool, device="cuda")
        for _, rows in self.experts():
            keep[rows] = False
        keep[self.end:] = False
        return keep

    def forward(self, act=P.ACT_NONE, save=False):
        out, z = (torch.full((self.R, self.N), MARK, dtype=BF16, device="cuda") for _ in range(2))
        P.osdp_expert_linear_fwd(self.x, self.plan, self.flat, 64, self.bias, self.T, self.k, self.E, self.N, self.K, act, out, z if save else None,
                                 self.ws(act, P.OP_LINEAR_FWD), check=True)
        return out, z

    def backward(self, act=P.ACT_NONE, dw_dtype=BF16, dw=None, flags=0, want_db=True):
        E, N, K = self.E, self.N, self.K
        dx = torch.full((self.R, K), MARK, dtype=BF16, device="cuda")
        if dw is None:
            dw = torch.full((E * N * K + 64,), MARK, dtype=dw_dtype, device="cuda")
        db = torch.full((E, N), math.nan, device="cuda") if want_db else None
        P.osdp_expert_linear_bwd(self.dy, self.x, self.plan, self.flat, 64, self.z if act else None, self.T, self.k, E, N, K, act, dx, dw, 64,
                                 P.DTYPE_FP32 if dw.dtype == torch.float32 else P.DTYPE_BF16, flags, db, self.ws(act, P.OP_LINEAR_BWD), check=True)
        return dx, dw, db

    def check_forward(self, act=P.ACT_NONE):
        out, z = self.forward(act, save=True)
        alone, untouched = self.forward(act)
        assert bool((untouched == MARK).all())
        assert torch.equal(alone[:self.end], out[:self.end])
        for v in (out, z):
            assert bool((v[self.end:] == MARK).all()) and bool((v[self.between()] == 0).all())
        for e, r in self.experts():
            x, w = self.x[r].to(D64), self.w[e].to(D64)
            want = x @ w.t()
            size = x.abs() @ w.abs().t()
            if self.bias is not None:
                want = want + self.bias[e].to(D64)
            # K products added in fp32 (the tensor core cuts what it adds: a whole unit), one rounding to bf16
            tol = (self.K + 2) * 2 * HALF32 * size + HALF32 * want.abs()
            assert bool(((z[r].to(D64) - want).abs() <= HALF16 * want.abs() + tol * (1 + HALF16)).all())
            # the activation's slope is at most 1.13; its tanh is good to 2^-10.9
            a = gelu(want, act)
            slack = 0.0 if act == P.ACT_NONE else 1.0
            assert bool(((out[r].to(D64) - a).abs() <= HALF16 * a.abs() + 1.2 * tol + slack * (0.5 * want.abs() * 2.0 ** -10 + 1e-6)).all())

    def check_backward(self, act=P.ACT_NONE, **kw):
        dx, dw, db = self.backward(act, **kw)
        assert bool((dx[self.end:] == MARK).all()) and bool((dx[self.between()] == 0).all())
        assert bool((dw[:64] == MARK).all())
        mine = dw[64:].view(self.E, self.N, self.K)
        out16 = HALF16 if dw.dtype == BF16 else HALF32
        for e in range(self.E):
            if not self.counts[e]:
                assert bool((mine[e] == 0).all()) and bool((db[e] == 0).all())
        for e, r in self.experts():
            g = self.dy[r].to(D64)
            if act:
                g = g * gelu_grad(self.z[r].to(D64), act)
            # G is rounded to bf16 as an operand (none without an activation), the derivative is good to 2^-18 of its largest terms
            off = 0.0 if act == P.ACT_NONE else HALF16 * (1 + HALF16)
            slip = 0.0 if act == P.ACT_NONE else 2.0 ** -18 * self.dy[r].to(D64).abs() * (1.0 + self.z[r].to(D64).abs())
            x, w, n = self.x[r].to(D64), self.w[e].to(D64), self.counts[e]
            ga = g.abs() + slip
            want, size = g @ w, ga @ w.abs()
            err = off * size + (slip @ w.abs() if act else 0.0)
            assert bool(((dx[r].to(D64) - want).abs() <= HALF16 * want.abs() + (1 + HALF16) * (err + (self.N + 2) * 2 * HALF32 * size)).all())
            want, size = g.t() @ x, ga.t() @ x.abs()
            err = off * size + (slip.t() @ x.abs() if act else 0.0)
            assert bool(((mine[e].to(D64) - want).abs() <= out16 * want.abs() + (1 + out16) * (err + (n + 66) * 2 * HALF32 * size)).all())
            want = g.sum(0)
            # sums of 8 rows, of 32 threads, of the tiles; each product rounded
            tol = (8 + 32 + n / 256 + 3) * HALF32 * ga.sum(0) + (slip.sum(0) if act else 0.0)
            assert bool(((db[e].to(D64) - want).abs() <= tol).all())


PRODUCTS = [(1, 2, 8, "even", 64, 64), (37, 2, 16, "skewed", 2064, 1032), (300, 3, 5, "holes", 136, 72), (9, 1, 1, "one", 8, 8),
            (1777, 2, 6, "skewed", 256, 520), (700, 2, 4, "one", 328, 264), (2500, 2, 3, "even", 1024, 512), (3000, 2, 4, "skewed", 2048, 1024),
            (200, 1, 300, "even", 72, 136), (5000, 2, 2, "holes", 4096, 1280)]


@pytest.mark.parametrize("act", [P.ACT_NONE, P.ACT_GELU_TANH, P.ACT_GELU_ERF])
@pytest.mark.parametrize("T,k,E,how,N,K", PRODUCTS)
def test_products_forward(T, k, E, how, N, K, act):
    Problem(T, k, E, how, N, K, bias=act != P.ACT_GELU_ERF).check_forward(act)


@pytest.mark.parametrize("act", [P.ACT_NONE, P.ACT_GELU_TANH, P.ACT_GELU_ERF])
@pytest.mark.parametrize("T,k,E,how,N,K", PRODUCTS)
def test_products_backward(T, k, E, how, N, K, act):
    Problem(T, k, E, how, N, K).check_backward(act, dw_dtype=torch.float32 if act == P.ACT_GELU_TANH else BF16)


@pytest.mark.parametrize("T", [5, 300])
def test_nobody_is_chosen(T):
    """Every choice is dropped: no row is written, and all gradients of the weights are zero."""
    p = Problem(T, 2, 6, "even", 136, 72)
    idx = torch.full((T, 2), 6, dtype=torch.int32, device="cuda")
    p.plan, p.pos, p.R = make_plan(idx, 6)
    out, _ = p.forward(P.ACT_GELU_TANH)
    assert p.R == len(out) and bool((out == MARK).all())
    dx, dw, db = p.backward(P.ACT_GELU_TANH)
    assert bool((dx == MARK).all()) and bool((dw[64:] == 0).all()) and bool((db == 0).all())


def test_gradients_are_added_and_left_out():
    p = Problem(300, 2, 5, "skewed", 264, 136)
    for dtype in (torch.float32, BF16):
        _, once, db = p.backward(dw_dtype=dtype)
        total = once.clone()
        total[64:] = 1.0
        p.backward(dw=total, flags=P.FLAG_ACCUMULATE_DW)
        half = HALF16 if dtype == BF16 else HALF32
        a, b = once[64:].to(D64), total[64:].to(D64)
        assert bool(((b - a - 1.0).abs() <= half * (a.abs() + b.abs())).all()) and bool((total[:64] == MARK).all())
    # each output alone has the bits that it has with the others
    dx, dw, db = p.backward()
    ws = p.ws(0, P.OP_LINEAR_BWD)
    alone = torch.full_like(dx, MARK)
    P.osdp_expert_linear_bwd(p.dy, None, p.plan, p.flat, 64, None, p.T, p.k, p.E, p.N, p.K, 0, alone, None, 0, 0, 0, None, ws, check=True)
    assert torch.equal(alone[:p.end], dx[:p.end])
    alone = torch.full_like(dw, MARK)
    P.osdp_expert_linear_bwd(p.dy, p.x, p.plan, None, 0, None, p.T, p.k, p.E, p.N, p.K, 0, None, alone, 64, 0, 0, None, ws, check=True)
    assert torch.equal(alone, dw)
    alone = torch.full_like(db, MARK)
    P.osdp_expert_linear_bwd(p.dy, None, p.plan, None, 0, None, p.T, p.k, p.E, p.N, p.K, 0, None, None, 0, 0, 0, alone, ws, check=True)
    assert torch.equal(alone, db)


def test_captured_calls_follow_the_choices():
    """One graph of plan, dispatch, product and gradients, replayed with other choices: nothing of them was kept."""
    T, k, E, N, K = 200, 2, 6, 136, 72
    p = Problem(T, k, E, "even", N, K)
    x = torch.randn(T, K, device="cuda").to(BF16)
    dout = torch.randn(T, N, device="cuda").to(BF16)
    w = torch.rand(T, k, device="cuda")
    idx = p.idx.clone()
    new = lambda *n: torch.zeros(*n, dtype=BF16, device="cuda")                      # noqa: E731
    xs, ys, dys, dxs, out = new(p.R, K), new(p.R, N), new(p.R, N), new(p.R, K), new(T, N)
    dw, dww = torch.zeros(E, N, K, device="cuda"), torch.zeros(T, k, device="cuda")
    wf, wb = p.ws(0, P.OP_LINEAR_FWD), p.ws(0, P.OP_LINEAR_BWD)

    def go():
        P.osdp_expert_plan(idx, T, k, E, p.plan, p.pos, check=True)
        P.osdp_expert_dispatch(x, p.plan, p.pos, None, None, T, k, E, K, xs, None, check=True)
        P.osdp_expert_linear_fwd(xs, p.plan, p.flat, 64, p.bias, T, k, E, N, K, 0, ys, None, wf, check=True)
        P.osdp_expert_combine(ys, p.plan, p.pos, w, T, k, E, N, out, check=True)
        P.osdp_expert_dispatch(dout, p.plan, p.pos, w, ys, T, k, E, N, dys, dww, check=True)
        P.osdp_expert_linear_bwd(dys, xs, p.plan, p.flat, 64, None, T, k, E, N, K, 0, dxs, dw, 0, P.DTYPE_FP32, 0, None, wb, check=True)
    go()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for how in ("one", "skewed", "even", "holes"):
        idx.copy_(choices(T, k, E, how, seed=5))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (out, dww, dw)]
        go()
        torch.cuda.synchronize()
        for a, b in zip(got, (out, dww, dw)):
            assert torch.equal(a, b), how
        i = idx.long()
        on = ((i >= 0) & (i < E)).to(D64)
        y = torch.einsum("tk,tjnk->tjn", x.to(D64), p.w.to(D64)[i.clamp(0, E - 1)]) + p.bias.to(D64)[i.clamp(0, E - 1)]
        want = (y * (w.to(D64) * on)[:, :, None]).sum(1)
        size = (y.abs() * (w.to(D64) * on)[:, :, None]).sum(1)
        # the products' rounding to bf16, the sum's, and fp32 sums of K
        assert bool(((out.to(D64) - want).abs() <= HALF16 * (1 + HALF16) * size + HALF16 * want.abs() + 1e-4).all()), how
    del graph


def test_status_word_stays_clear():
    p = Problem(500, 2, 4, "skewed", 512, 256)
    ws = p.ws(P.ACT_GELU_TANH, P.OP_LINEAR_BWD)
    out = torch.empty(p.R, p.N, dtype=BF16, device="cuda")
    P.osdp_expert_linear_fwd(p.x, p.plan, p.flat, 64, p.bias, p.T, p.k, p.E, p.N, p.K, P.ACT_GELU_TANH, out, None, ws, check=True)
    assert P.osdp_read_device_status(ws) == (0, 0)
