"""What the block norm, the optimiser step and the int8 layer refuse, and their host-side layouts.  No GPU: every check
stands before the first launch, so made-up addresses are never read."""
import ctypes

import pytest

import paper_2209_13258_b200 as P

A = 1 << 20        # aligned to everything that is asked for
NULL, SHAPE, SPLIT, ALIGN, WS, UNSUPPORTED = 1, 2, 3, 4, 5, 6


def fwd(x=A, y=A, M=4, D=64, rt=0, post=1, w_post=A, b_post=None, eps_post=1e-5, gate=A, alpha=1.0, beta=1.0, pre=1, w_pre=A, b_pre=None,
        eps_pre=1e-5, r=A, u=A, u_scale=None, stats=A):
    return P.osdp_block_norm_fwd(x, y, M, D, rt, post, w_post, b_post, eps_post, gate, alpha, beta, pre, w_pre, b_pre, eps_pre, r, u, u_scale,
                                 stats, stream=0)


@pytest.mark.parametrize("change,want", [
    ({"x": None}, NULL), ({"u": None}, NULL), ({"r": None, "pre": 0, "u": None}, NULL),
    ({"M": -1}, SHAPE), ({"D": 0}, SHAPE), ({"M": 1 << 40}, SHAPE), ({"D": 60}, ALIGN), ({"D": 16392}, UNSUPPORTED),
    ({"rt": 2}, UNSUPPORTED), ({"post": 3}, UNSUPPORTED), ({"pre": -1}, UNSUPPORTED), ({"b_post": A}, UNSUPPORTED), ({"b_pre": A}, UNSUPPORTED),
    ({"alpha": float("nan")}, UNSUPPORTED), ({"beta": float("inf")}, UNSUPPORTED), ({"eps_pre": -1.0}, UNSUPPORTED),
    ({"eps_post": float("nan")}, UNSUPPORTED),
    ({"x": A + 8}, ALIGN), ({"x": A + 16, "rt": 1}, ALIGN), ({"y": A + 2}, ALIGN), ({"u": A + 8}, ALIGN), ({"u": A + 4, "u_scale": A}, ALIGN),
    ({"gate": A + 4}, ALIGN), ({"stats": A + 8}, ALIGN), ({"w_pre": A + 8}, ALIGN)])
def test_block_norm_forward_refuses(change, want):
    assert fwd(**change) == want


def test_block_norm_of_no_rows_is_nothing():
    assert fwd(M=0) == 0 and fwd(M=0, x=None, y=None, r=None, u=None, stats=None) == 0


def bwd(dr=A, du=A, y=A, r=A, stats=A, M=4, D=64, rt=0, post=1, w_post=A, b_post=None, gate=A, alpha=1.0, beta=1.0, pre=1, w_pre=A, dx=A, dy=A,
        dw_post=A, db_post=None, dgate=A, dw_pre=A, db_pre=None, ws=(A, 1 << 30)):
    return P.osdp_block_norm_bwd(dr, du, y, r, stats, M, D, rt, post, w_post, b_post, gate, alpha, beta, pre, w_pre, dx, dy, dw_post, db_post,
                                 dgate, dw_pre, db_pre, ws, stream=0)


@pytest.mark.parametrize("change,want", [
    ({"du": None}, NULL), ({"r": None}, NULL), ({"stats": None}, NULL), ({"y": None}, NULL), ({"ws": None}, NULL),
    ({"pre": 0, "dr": None, "dw_pre": None}, NULL),
    ({"M": -2}, SHAPE), ({"D": 12}, ALIGN), ({"D": 1 << 20}, UNSUPPORTED), ({"rt": 7}, UNSUPPORTED), ({"db_post": A}, UNSUPPORTED),
    ({"db_pre": A}, UNSUPPORTED), ({"post": 0}, UNSUPPORTED), ({"pre": 0}, UNSUPPORTED), ({"alpha": float("inf")}, UNSUPPORTED),
    ({"dy": A + 8}, ALIGN), ({"dx": A + 16, "rt": 1}, ALIGN), ({"dgate": A + 2}, ALIGN), ({"ws": (A + 16, 1 << 30)}, ALIGN), ({"ws": (A, 4096)}, WS)])
def test_block_norm_backward_refuses(change, want):
    assert bwd(**change) == want


def test_block_norm_workspace():
    assert P.osdp_block_norm_workspace_bytes(0, 64)[0] == 0
    n = [P.osdp_block_norm_workspace_bytes(M, 4096)[1] for M in (1, 100000)]
    assert n[0] == n[1] >= 4 * 4 * 4096
    assert P.osdp_block_norm_workspace_bytes(1, 63)[0] == ALIGN and P.osdp_block_norm_workspace_bytes(-1, 64)[0] == SHAPE


def tensors(n=1, **kw):
    a = (P.AdamWTensor * max(n, 1))()
    for i in range(n):
        a[i].param, a[i].grad, a[i].numel, a[i].state_offset, a[i].lr, a[i].weight_decay = A, A, 100, 256 * i, 1e-3, 0.0
        for k, v in kw.items():
            setattr(a[i], k, v)
    return a


def step(t=None, n=1, pt=1, st=1, master=None, m=A, v=A, sm=A, sv=A, b1=0.9, b2=0.999, eps=1e-8, at=1, clip=None):
    return P.osdp_adamw_step(tensors() if t is None else t, n, pt, st, master, m, v, sm, sv, b1, b2, eps, at, clip, stream=0)


@pytest.mark.parametrize("change,want", [
    ({"n": -1}, SHAPE), ({"pt": 2}, UNSUPPORTED), ({"st": 0}, UNSUPPORTED), ({"m": None}, NULL), ({"v": None}, NULL),
    ({"st": 2, "sm": None}, NULL), ({"m": A + 16}, ALIGN), ({"master": A, "pt": 1}, UNSUPPORTED), ({"master": A + 4, "pt": 0}, ALIGN),
    ({"b1": 1.0}, UNSUPPORTED), ({"b2": -0.1}, UNSUPPORTED), ({"eps": -1.0}, UNSUPPORTED), ({"eps": float("nan")}, UNSUPPORTED),
    ({"at": 0}, UNSUPPORTED), ({"clip": A + 2}, ALIGN),
    ({"t": tensors(param=None)}, NULL), ({"t": tensors(grad=None)}, NULL), ({"t": tensors(numel=-1)}, SHAPE), ({"t": tensors(numel=1 << 50)}, SHAPE),
    ({"t": tensors(state_offset=100)}, ALIGN), ({"t": tensors(state_offset=-256)}, ALIGN), ({"t": tensors(param=A + 2)}, ALIGN),
    ({"t": tensors(grad=A + 1), "pt": 0}, ALIGN), ({"t": tensors(lr=float("nan"))}, UNSUPPORTED), ({"t": tensors(weight_decay=float("inf"))}, UNSUPPORTED)])
def test_step_refuses(change, want):
    assert step(**change) == want


def test_step_over_nothing():
    assert step(n=0) == 0
    assert step(t=tensors(numel=0), m=None, v=None) == 0
    assert P.osdp_adamw_step(None, 1, 1, 1, None, A, A, A, A, 0.9, 0.99, 1e-8, 1, None, stream=0) == NULL


def test_gradient_norm_refuses():
    need = P.osdp_grad_norm_workspace_bytes(3)[1]
    go = lambda t=None, n=1, dt=1, mx=1.0, out=A, ws=(A, need): P.osdp_grad_norm(tensors() if t is None else t, n, dt, mx, out, ws, stream=0)  # noqa: E731
    assert go(out=None) == NULL and go(ws=None) == NULL and go(ws=(A + 8, need)) == ALIGN and go(ws=(A, 256)) == WS
    assert go(dt=2) == UNSUPPORTED and go(mx=float("nan")) == UNSUPPORTED and go(n=-1) == SHAPE and go(t=tensors(grad=None)) == NULL
    assert P.osdp_grad_norm_workspace_bytes(-1)[0] == SHAPE
    assert P.osdp_grad_norm_workspace_bytes(5000)[1] > need


def test_state_layout():
    assert P.osdp_adamw_layout([1, 256, 257, 0, 5]) == (0, [0, 256, 512, 1024, 1024], 1280)
    assert P.osdp_adamw_layout([]) == (0, [], 0)
    assert P.osdp_adamw_layout([-1])[0] == SHAPE and P.osdp_adamw_layout([1 << 43])[0] == SHAPE
    assert ctypes.sizeof(P.AdamWTensor) == 48


def i8(x=A, sx=A, w=A, off=0, sw=A, b=None, M=4, N=64, K=64, k=1, split=0, act=0, out=A, ws=(A, 256)):
    return P.osdp_split_linear_fwd_i8(x, sx, w, off, sw, b, M, N, K, k, split, act, out, ws, stream=0)


@pytest.mark.parametrize("change,want", [
    ({"x": None}, NULL), ({"w": None}, NULL), ({"sw": None}, NULL), ({"out": None}, NULL), ({"ws": None}, NULL),
    ({"M": -1}, SHAPE), ({"N": 0}, SHAPE), ({"K": 131072}, SHAPE), ({"K": 72}, ALIGN), ({"N": 60}, ALIGN), ({"off": 8}, ALIGN), ({"off": -16}, ALIGN),
    ({"k": 2, "split": 1, "K": 80}, ALIGN), ({"k": 2, "N": 72}, ALIGN), ({"k": 100}, SPLIT), ({"k": -1}, SPLIT), ({"split": 2}, SPLIT),
    ({"act": 3}, UNSUPPORTED), ({"x": A + 8}, ALIGN), ({"out": A + 2}, ALIGN), ({"b": A + 4}, ALIGN), ({"ws": (A + 64, 256)}, ALIGN),
    ({"ws": (A, 128)}, WS), ({"sx": None}, WS)])
def test_int8_refuses(change, want):
    assert i8(**change) == want


def test_int8_of_no_tokens_and_quantiser():
    assert i8(M=0) == 0
    q = lambda x=A, M=4, K=64, c=A, s=A: P.osdp_quantize_rows_i8(x, M, K, c, s, stream=0)      # noqa: E731
    assert q(M=0) == 0 and q(M=-1) == SHAPE and q(K=0) == SHAPE and q(K=1 << 20) == SHAPE and q(K=12) == ALIGN
    assert q(x=None) == NULL and q(c=None) == NULL and q(s=None) == NULL and q(x=A + 8) == ALIGN and q(c=A + 4) == ALIGN
    assert P.osdp_i8_workspace_bytes(10, 64) == (0, 256 + 256 + 640)
    assert P.osdp_i8_workspace_bytes(10, 0)[0] == SHAPE
