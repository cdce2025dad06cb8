"""What routing, the experts' rows and the experts' products refuse, and their host-side sizes.  No GPU: every check stands
before the first launch, so made-up addresses are never read."""
import pytest
import torch

import paper_2209_13258_b200 as P
from paper_2209_13258_b200 import nn as pnn

A = 1 << 20
NULL, SHAPE, ALIGN, WS, UNSUPPORTED = 1, 2, 4, 5, 6
NAN, INF = float("nan"), float("inf")


def route(logits=A, ld=16, dt=1, bias=None, T=4, E=16, k=2, score=0, groups=1, top=1, take=1, renorm=1, scale=1.0, idx=A, w=A):
    return P.osdp_route_fwd(logits, ld, dt, bias, T, E, k, score, groups, top, take, renorm, scale, idx, w, stream=0)


@pytest.mark.parametrize("change,want", [
    ({"logits": None}, NULL), ({"idx": None}, NULL), ({"w": None}, NULL), ({"T": -1}, SHAPE), ({"E": 0}, SHAPE), ({"E": 1025, "ld": 2000}, SHAPE),
    ({"k": 0}, SHAPE), ({"k": 17}, SHAPE), ({"E": 1, "k": 2}, SHAPE), ({"ld": 15}, SHAPE), ({"T": 1 << 40}, SHAPE), ({"T": 1 << 30}, SHAPE),
    ({"groups": 3}, SHAPE), ({"groups": 0}, SHAPE), ({"groups": 4, "top": 5}, SHAPE), ({"groups": 4, "top": 0}, SHAPE), ({"groups": 16, "top": 1}, SHAPE),
    ({"E": 64, "ld": 64, "groups": 64, "top": 64}, SHAPE), ({"take": 0}, UNSUPPORTED), ({"take": 3}, UNSUPPORTED), ({"dt": 2}, UNSUPPORTED),
    ({"score": 2}, UNSUPPORTED), ({"scale": NAN}, UNSUPPORTED), ({"scale": INF}, UNSUPPORTED), ({"scale": 1e300}, UNSUPPORTED), ({"logits": A + 2}, ALIGN),
    ({"logits": A + 1, "dt": 0}, ALIGN), ({"bias": A + 2}, ALIGN), ({"idx": A + 1}, ALIGN), ({"w": A + 2}, ALIGN)])
def test_route_refuses(change, want):
    assert route(**change) == want


def route_bwd(dw=A, logits=A, ld=16, dt=1, idx=A, T=4, E=16, k=2, score=0, renorm=1, scale=1.0, out=A, ld_out=16):
    return P.osdp_route_bwd(dw, logits, ld, dt, idx, T, E, k, score, renorm, scale, out, ld_out, stream=0)


@pytest.mark.parametrize("change,want", [
    ({"dw": None}, NULL), ({"logits": None}, NULL), ({"idx": None}, NULL), ({"out": None}, NULL), ({"ld_out": 15}, SHAPE), ({"ld": 3}, SHAPE), ({"T": -1}, SHAPE),
    ({"k": 17}, SHAPE), ({"dt": 3}, UNSUPPORTED), ({"score": -1}, UNSUPPORTED), ({"scale": NAN}, UNSUPPORTED), ({"out": A + 2}, ALIGN), ({"dw": A + 1}, ALIGN)])
def test_route_backward_refuses(change, want):
    assert route_bwd(**change) == want


def test_routing_of_no_tokens_is_nothing():
    assert route(T=0, logits=None, idx=None, w=None) == 0 and route_bwd(T=0, dw=None, logits=None, idx=None, out=None) == 0


def test_rows():
    assert P.osdp_expert_rows(0, 2, 8)[:2] == (0, 0)
    assert P.osdp_expert_rows(1, 2, 8)[:2] == (0, 128) and P.osdp_expert_rows(1, 1, 8)[:2] == (0, 64)
    # enough for every spread of the choices: the worst has 1 (mod 64) rows for each expert
    for T, k, E in ((7, 2, 3), (100, 4, 60), (1000, 1, 1000), (64, 1, 1), (129, 3, 3)):
        n, rows = T * k, P.osdp_expert_rows(T, k, E)[1]
        used = min(n, E)
        worst = max((-(-(n - m + 1) // 64) + m - 1) * 64 for m in range(1, used + 1))
        assert worst <= rows < worst + 64 * used and rows % 64 == 0
    assert P.osdp_expert_rows(1, 2, 8)[2] >= 5 * 8 + 4
    for bad in ((-1, 2, 8), (1, 0, 8), (1, 9, 8), (1, 2, 0), (1, 2, 2000), (1 << 30, 2, 8)):
        assert P.osdp_expert_rows(*bad)[0] == SHAPE


def test_plan_and_rows_refuse():
    plan = lambda idx=A, T=4, k=2, E=8, p=A, pos=A: P.osdp_expert_plan(idx, T, k, E, p, pos, stream=0)             # noqa: E731
    assert plan(idx=None) == NULL and plan(p=None) == NULL and plan(pos=None) == NULL and plan(T=-1) == SHAPE and plan(p=A + 4) == ALIGN and plan(pos=A + 2) == ALIGN
    d = lambda x=A, p=A, pos=A, w=None, y=None, T=4, k=2, E=8, D=64, r=A, dw=None: P.osdp_expert_dispatch(x, p, pos, w, y, T, k, E, D, r, dw, stream=0)   # noqa: E731
    assert d(x=None) == NULL and d(p=None) == NULL and d(pos=None) == NULL and d(r=None) == NULL and d(dw=A) == NULL
    assert d(D=0) == SHAPE and d(D=12) == ALIGN and d(D=1 << 20) == SHAPE and d(k=9) == SHAPE and d(T=0) == 0 and d(T=0, x=None, r=None) == 0
    assert d(x=A + 8) == ALIGN and d(r=A + 8) == ALIGN and d(w=A + 1) == ALIGN and d(y=A + 8, dw=A) == ALIGN
    c = lambda r=A, p=A, pos=A, w=None, T=4, k=2, E=8, D=64, o=A: P.osdp_expert_combine(r, p, pos, w, T, k, E, D, o, stream=0)             # noqa: E731
    assert c(r=None) == NULL and c(p=None) == NULL and c(pos=None) == NULL and c(o=None) == NULL and c(D=4) == ALIGN and c(o=A + 8) == ALIGN and c(T=0) == 0
    assert c(E=0) == SHAPE and c(D=-8) == SHAPE


def fwd(rows=A, plan=A, w=A, off=0, bias=None, T=100, k=2, E=8, N=64, K=64, act=0, out=A, z=None, ws=(A, 256)):
    return P.osdp_expert_linear_fwd(rows, plan, w, off, bias, T, k, E, N, K, act, out, z, ws, stream=0)


@pytest.mark.parametrize("change,want", [
    ({"rows": None}, NULL), ({"plan": None}, NULL), ({"w": None}, NULL), ({"out": None}, NULL), ({"ws": None}, NULL), ({"T": -1}, SHAPE), ({"N": 0}, SHAPE),
    ({"K": -8}, SHAPE), ({"N": 1 << 25}, SHAPE), ({"N": 60}, ALIGN), ({"K": 4}, ALIGN), ({"act": 3}, UNSUPPORTED), ({"off": 4}, ALIGN), ({"off": -8}, ALIGN),
    ({"rows": A + 8}, ALIGN), ({"out": A + 8}, ALIGN), ({"z": A + 2}, ALIGN), ({"bias": A + 4}, ALIGN), ({"ws": (A + 64, 256)}, ALIGN), ({"ws": (A, 128)}, WS),
    ({"k": 17}, SHAPE), ({"E": 0}, SHAPE)])
def test_products_refuse(change, want):
    assert fwd(**change) == want


def bwd(dy=A, rows=A, plan=A, w=A, off=0, z=None, T=100, k=2, E=8, N=64, K=64, act=0, dx=A, dw=A, dw_off=0, dt=0, flags=0, db=A, ws=(A, 1 << 30)):
    return P.osdp_expert_linear_bwd(dy, rows, plan, w, off, z, T, k, E, N, K, act, dx, dw, dw_off, dt, flags, db, ws, stream=0)


@pytest.mark.parametrize("change,want", [
    ({"dy": None}, NULL), ({"rows": None}, NULL), ({"plan": None}, NULL), ({"w": None}, NULL), ({"act": 1}, NULL), ({"ws": None}, NULL), ({"ws": (A, 2560)}, WS),
    ({"dt": 2}, UNSUPPORTED), ({"flags": 2}, UNSUPPORTED), ({"act": 5}, UNSUPPORTED), ({"dw_off": 4}, ALIGN), ({"dw": A + 8}, ALIGN), ({"db": A + 4}, ALIGN),
    ({"dx": A + 2}, ALIGN), ({"dy": A + 8}, ALIGN), ({"N": 4}, ALIGN), ({"K": 0}, SHAPE)])
def test_products_backward_refuse(change, want):
    assert bwd(**change) == want


def test_products_workspace():
    size = lambda act=0, op=P.OP_LINEAR_BWD, T=100, N=64: P.osdp_expert_linear_workspace_bytes(T, 2, 8, N, 64, act, op)       # noqa: E731
    assert size(op=P.OP_LINEAR_FWD) == (0, 256)
    rows = P.osdp_expert_rows(100, 2, 8)[1]
    assert size(act=1)[1] - size()[1] == rows * 64 * 2 and size()[1] >= 256 + rows // 64 * 64 * 4
    assert size(op=P.OP_MLP_FWD)[0] == UNSUPPORTED and size(act=7)[0] == UNSUPPORTED and size(N=12)[0] == ALIGN and size(T=-1)[0] == SHAPE
    assert size(T=0) == (0, 256)


def test_router_module_refuses():
    mk = lambda **kw: pnn.ExpertRouter(**{"experts": 16, "top_k": 2, "device": "cpu", **kw})      # noqa: E731
    for bad in ({"experts": 0}, {"experts": 2000}, {"top_k": 0}, {"top_k": 17}, {"experts": 4, "top_k": 5}, {"score": "relu"}, {"groups": 3}, {"groups": 0},
                {"groups": 8, "top_groups": 9}, {"groups": 16, "top_groups": 1}, {"group_take": 3}):
        with pytest.raises(ValueError):
            mk(**bad)
    r = mk(bias=True)
    assert r.bias.shape == (16,) and "bias" in r.state_dict() and mk().bias is None
    with pytest.raises(RuntimeError):
        r(torch.zeros(4, 16))


def test_mlp_module_refuses():
    for bad in ((60, 64, 4), (64, 12, 4), (64, 64, 0), (64, 64, 2000), (0, 64, 4)):
        with pytest.raises(ValueError):
            pnn.ExpertMLP(*bad, device="cpu")
    m = pnn.ExpertMLP(16, 24, 3, device="cpu")
    assert m.w1.shape == (3, 24, 16) and m.w2.shape == (3, 16, 24) and m.b1.shape == (3, 24) and m.b2.shape == (3, 16)
    assert "_status" not in m.state_dict()
    with pytest.raises(RuntimeError):
        m(torch.zeros(4, 16, dtype=torch.bfloat16), torch.zeros(4, 2), torch.zeros(4, 2, dtype=torch.int32))


def test_calls_as_words():
    """The binding packs its arguments; what the packed entry point itself refuses, and that integers are not cut."""
    import struct
    from paper_2209_13258_b200 import binding as B
    call = B.lib().osdp_call
    assert call(None) == NULL
    for which in (-1, 7, 1 << 40):
        assert call(struct.pack("=25q", which, *[0] * 24)) == UNSUPPORTED
    assert route(k=(1 << 32) + 2) == SHAPE and route(score=1 << 32) == UNSUPPORTED and fwd(k=(1 << 32) + 2) == SHAPE and bwd(flags=1 << 32) == UNSUPPORTED
    with pytest.raises(struct.error):
        route(T=1 << 64)
    with pytest.raises(P.OsdpError):
        P.osdp_expert_plan(None, 4, 2, 8, A, A, stream=0, check=True)


def test_rows_in_an_expert_order():
    assert P.EXPERT_ROWS == 64 and P.MAX_EXPERTS == 1024 and P.MAX_TOP_K == 16
