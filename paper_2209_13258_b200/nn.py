"""torch.nn front end of the split linear layer: a module whose forward and backward are the library's
calls (Section 3.3: the operator is processed as k sequential slices), so that a model can swap an
``nn.Linear`` for it the way the paper's wrapper replaces FSDP's.

Only argument marshalling and autograd bookkeeping happen here; every product, sum and activation runs in
the CUDA kernels behind ``osdp_split_linear_fwd`` / ``osdp_split_linear_bwd``.  CUDA only: there is no CPU path.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding as B


def _check_fp32(device, **vectors):
    """name=(tensor or None, elements).  The kernels read these as fp32 from the address alone: another dtype, device or
    length would be misread, and read beyond its end."""
    for name, (v, n) in vectors.items():
        if v is None:
            continue
        if v.dtype is not torch.float32:
            raise TypeError("%s is %s and has to be fp32: module.to(dtype) casts every floating-point parameter and buffer" % (name, v.dtype))
        if v.device != device:
            raise RuntimeError("%s is on %s and its input on %s: they have to be on one CUDA device" % (name, v.device, device))
        if v.numel() != n or not v.is_contiguous():
            raise ValueError("%s has to be contiguous with %d elements" % (name, n))


def _elsewhere(x):
    """Whether x is on another CUDA device than the current one, on whose current stream a call launches."""
    return x.is_cuda and x.get_device() != torch.cuda.current_device()


def _check_flat(device, flat, numel):
    if flat.dtype is not torch.bfloat16:
        raise TypeError("the flat parameter buffer is %s and has to be bf16" % flat.dtype)
    if flat.device != device:
        raise RuntimeError("the flat parameter buffer is on %s and its input on %s: they have to be on one CUDA device" % (flat.device, device))
    if flat.numel() < numel or not flat.is_contiguous():
        raise ValueError("the flat parameter buffer has to be contiguous with %d elements" % numel)


class _SplitLinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, layer):
        M = x.numel() // layer.in_features
        x2 = x.reshape(M, layer.in_features)
        if not x2.is_contiguous():
            x2 = x2.contiguous()
        N, K, k = layer.out_features, layer.in_features, layer.k_split
        out = torch.empty(M, N, dtype=torch.bfloat16, device=x.device)
        # any gradient of an activated layer, the bias gradient included, is taken through act'(Z)
        need_z = layer.act != B.ACT_NONE and (x.requires_grad or weight.requires_grad or
                                              (bias is not None and bias.requires_grad))
        z = torch.empty(M, N, dtype=torch.bfloat16, device=x.device) if need_z else None
        ws = layer._workspace(M)
        # the parameter is read in place from the flat buffer it lives in (element offset of the view)
        B.osdp_split_linear_fwd(x2, layer.flat, layer.w_offset, bias, M, N, K, k, layer.split_dim, layer.act, out, z, ws,
                                check=True, flags=layer.flags)
        ctx.layer, ctx.M = layer, M
        ctx.save_for_backward(x2, z if z is not None else torch.empty(0, device=x.device), weight)
        ctx.x_shape = x.shape
        ctx.has_bias = bias is not None
        return out.reshape(*x.shape[:-1], N)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        layer, M = ctx.layer, ctx.M
        x2, z, weight = ctx.saved_tensors
        N, K, k = layer.out_features, layer.in_features, layer.k_split
        dy2 = dy.reshape(M, N)
        if not dy2.is_contiguous():
            dy2 = dy2.contiguous()
        need_dx, need_dw, need_db = ctx.needs_input_grad[0], ctx.needs_input_grad[1], ctx.has_bias and ctx.needs_input_grad[2]
        dx = torch.empty(M, K, dtype=torch.bfloat16, device=dy.device) if need_dx else None
        dw = torch.empty(N, K, dtype=torch.bfloat16, device=dy.device) if need_dw else None
        db = torch.empty(N, dtype=torch.float32, device=dy.device) if need_db else None
        ws = layer._workspace(M)
        B.osdp_split_linear_bwd(dy2, x2, layer.flat, layer.w_offset, z if z.numel() else None, M, N, K, k,
                                layer.split_dim, layer.act, dx, dw, 0, B.DTYPE_BF16, layer.flags & B.FLAG_CARRY_BF16,
                                db, ws, check=True)
        return (dx.reshape(ctx.x_shape) if need_dx else None), dw, db, None


class SplitLinear(torch.nn.Module):
    """y = act(x W^T + b), computed as `k_split` sequential slices of W along `split_dim`
    (SPLIT_OUT: rows of W, SPLIT_RED: columns of W and x).  bf16 activations and weight, fp32 bias.

    `flat` (optional): a 1-D bf16 parameter buffer that already holds W [out_features, in_features] row-major
    at element offset `w_offset` (a multiple of 8); the module's `weight` is then a view of it and nothing is
    copied, which is how a flat-parameter wrapper stores its layers.  Without it the module owns its buffer.
    """

    def __init__(self, in_features, out_features, bias=True, k_split=1, split_dim=B.SPLIT_OUT, act=B.ACT_NONE,
                 flags=0, flat=None, w_offset=0, device="cuda"):
        super().__init__()
        if in_features % 8 or out_features % 8:
            raise ValueError("in_features and out_features must be multiples of 8")
        self.in_features, self.out_features = int(in_features), int(out_features)
        self.k_split, self.split_dim, self.act, self.flags = int(k_split), int(split_dim), int(act), int(flags)
        n = self.in_features * self.out_features
        if flat is None:
            w = torch.empty(n, dtype=torch.bfloat16, device=device)
            torch.nn.init.normal_(w, std=0.02)
            self.flat_param = torch.nn.Parameter(w)
            self._flat_owner, self.w_offset = None, 0
        else:
            if flat.dtype != torch.bfloat16 or flat.dim() != 1 or w_offset % 8 or w_offset + n > flat.numel():
                raise ValueError("flat must be a 1-D bf16 buffer holding W at a multiple-of-8 element offset")
            self.flat_param = None
            self._flat_owner, self.w_offset = flat, int(w_offset)
        self.bias = torch.nn.Parameter(torch.zeros(self.out_features, dtype=torch.float32, device=device)) if bias else None
        self._ws = None
        rc, _ = B.osdp_split_linear_workspace_bytes(1, self.out_features, self.in_features, self.k_split, self.split_dim,
                                                    self.act, B.OP_LINEAR_FWD, self.flags)
        if rc:
            raise B.OsdpError(rc, "SplitLinear")

    @property
    def flat(self):
        return self.flat_param if self._flat_owner is None else self._flat_owner

    @property
    def weight(self):
        n = self.in_features * self.out_features
        return self.flat[self.w_offset:self.w_offset + n].view(self.out_features, self.in_features)

    def _workspace(self, M):
        need = 0
        for op in (B.OP_LINEAR_FWD, B.OP_LINEAR_BWD):
            rc, n = B.osdp_split_linear_workspace_bytes(M, self.out_features, self.in_features, self.k_split,
                                                        self.split_dim, self.act, op, self.flags)
            if rc:
                raise B.OsdpError(rc, "osdp_split_linear_workspace_bytes")
            need = max(need, n)
        if self._ws is None or self._ws.numel() < need or self._ws.device != self.flat.device:
            self._ws = B.new_workspace(need, device=self.flat.device)
        return self._ws

    def forward(self, x):
        if not x.is_cuda:
            raise RuntimeError("SplitLinear runs on CUDA only: there is no CPU path")
        if x.dtype != torch.bfloat16:
            raise TypeError("SplitLinear takes bf16 activations")
        _check_flat(x.device, self.flat, self.w_offset + self.in_features * self.out_features)
        _check_fp32(x.device, bias=(self.bias, self.out_features))
        return _SplitLinearFn.apply(x, self.weight, self.bias, self)


class _SplitMLPFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, flat, b1, b2, layer):
        H, F, k = layer.hidden, layer.ffn, layer.k_split
        M = x.numel() // H
        x2 = x.reshape(M, H)
        if not x2.is_contiguous():
            x2 = x2.contiguous()
        out = torch.empty(M, H, dtype=torch.bfloat16, device=x.device)
        need_grad = x.requires_grad or flat.requires_grad
        # with recomputation no [M, ffn] activation is kept between forward and backward
        z1 = torch.empty(M, F, dtype=torch.bfloat16, device=x.device) if need_grad and not layer.recompute else None
        ws = layer._workspace(M)
        B.osdp_split_mlp_fwd(x2, layer.flat, layer.off_w1, b1, layer.off_w2, b2, M, H, F, k, layer.act, out, z1, ws,
                             check=True, flags=layer.flags & B.FLAG_CARRY_BF16)
        ctx.layer, ctx.M, ctx.x_shape = layer, M, x.shape
        ctx.has_b = (b1 is not None, b2 is not None)
        empty = torch.empty(0, device=x.device)
        ctx.save_for_backward(x2, z1 if z1 is not None else empty, b1 if b1 is not None else empty)
        return out.reshape(*x.shape[:-1], H)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        layer, M = ctx.layer, ctx.M
        H, F, k = layer.hidden, layer.ffn, layer.k_split
        x2, z1, b1 = ctx.saved_tensors
        dy2 = dy.reshape(M, H)
        if not dy2.is_contiguous():
            dy2 = dy2.contiguous()
        need_dx, need_dw = ctx.needs_input_grad[0], ctx.needs_input_grad[1]
        dx = torch.empty(M, H, dtype=torch.bfloat16, device=dy.device) if need_dx else None
        # the gradient of the flat parameter buffer, laid out like it: dW1 and dW2 at the offsets of W1 and W2
        dflat = torch.zeros_like(layer.flat) if need_dw else None
        db1 = torch.empty(F, dtype=torch.float32, device=dy.device) if ctx.has_b[0] and ctx.needs_input_grad[2] else None
        db2 = torch.empty(H, dtype=torch.float32, device=dy.device) if ctx.has_b[1] and ctx.needs_input_grad[3] else None
        flags = (layer.flags & B.FLAG_CARRY_BF16) | (B.FLAG_RECOMPUTE if layer.recompute else 0)
        ws = layer._workspace(M)
        B.osdp_split_mlp_bwd(dy2, x2, layer.flat, layer.off_w1, layer.off_w2, z1 if z1.numel() else None, M, H, F, k,
                             layer.act, dx, dflat, layer.off_w1, layer.off_w2, B.DTYPE_BF16, flags, db1, db2, ws,
                             check=True, b1=b1 if b1.numel() else None)
        return (dx.reshape(ctx.x_shape) if need_dx else None), dflat, db1, db2, None


class SplitMLP(torch.nn.Module):
    """y = act(x W1^T + b1) W2^T + b2, the transformer MLP block computed as `k_split` sequential slices of the
    ffn dimension (Section 3.3 applied to both MatMuls: the first layer's output slice feeds the second layer's
    reduction slice, so only an [M, ffn / k] intermediate exists at a time).  W1 [ffn, hidden] and W2 [hidden, ffn]
    live in one flat bf16 parameter buffer (`flat_param`, W1 first), biases are fp32.

    recompute=True is the activation-checkpointing setting of Section 2.3: the forward saves no [M, ffn]
    pre-activation and the backward recomputes it slice by slice.
    """

    def __init__(self, hidden, ffn, bias=True, k_split=1, act=B.ACT_GELU_TANH, recompute=False, flags=0, device="cuda"):
        super().__init__()
        if hidden % 8 or ffn % 8:
            raise ValueError("hidden and ffn must be multiples of 8")
        self.hidden, self.ffn, self.k_split, self.act = int(hidden), int(ffn), int(k_split), int(act)
        self.recompute, self.flags = bool(recompute), int(flags)
        self.off_w1, self.off_w2 = 0, self.hidden * self.ffn
        w = torch.empty(2 * self.hidden * self.ffn, dtype=torch.bfloat16, device=device)
        torch.nn.init.normal_(w, std=0.02)
        self.flat_param = torch.nn.Parameter(w)
        mk = lambda n: torch.nn.Parameter(torch.zeros(n, dtype=torch.float32, device=device)) if bias else None
        self.b1, self.b2 = mk(self.ffn), mk(self.hidden)
        self._ws = None
        rc, _ = B.osdp_split_linear_workspace_bytes(1, self.ffn, self.hidden, self.k_split, B.SPLIT_OUT, self.act,
                                                    B.OP_MLP_FWD, self.flags)
        if rc:
            raise B.OsdpError(rc, "SplitMLP")

    @property
    def flat(self):
        return self.flat_param

    @property
    def w1(self):
        return self.flat_param[:self.off_w2].view(self.ffn, self.hidden)

    @property
    def w2(self):
        return self.flat_param[self.off_w2:].view(self.hidden, self.ffn)

    def _workspace(self, M):
        need = 0
        for op, fl in ((B.OP_MLP_FWD, self.flags & B.FLAG_CARRY_BF16),
                       (B.OP_MLP_BWD, (self.flags & B.FLAG_CARRY_BF16) | (B.FLAG_RECOMPUTE if self.recompute else 0))):
            rc, n = B.osdp_split_linear_workspace_bytes(M, self.ffn, self.hidden, self.k_split, B.SPLIT_OUT, self.act,
                                                        op, fl)
            if rc:
                raise B.OsdpError(rc, "osdp_split_linear_workspace_bytes")
            need = max(need, n)
        if self._ws is None or self._ws.numel() < need or self._ws.device != self.flat.device:
            self._ws = B.new_workspace(need, device=self.flat.device)
        return self._ws

    def forward(self, x):
        if not x.is_cuda:
            raise RuntimeError("SplitMLP runs on CUDA only: there is no CPU path")
        if x.dtype != torch.bfloat16:
            raise TypeError("SplitMLP takes bf16 activations")
        _check_flat(x.device, self.flat_param, 2 * self.hidden * self.ffn)
        _check_fp32(x.device, b1=(self.b1, self.ffn), b2=(self.b2, self.hidden))
        return _SplitMLPFn.apply(x, self.flat_param, self.b1, self.b2, self)


class _ZdpLinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, shard, bias, layer, *dp_parts):
        impl = layer.impl
        M = x.numel() // impl.K
        x2 = x.reshape(M, impl.K)
        if not x2.is_contiguous():
            x2 = x2.contiguous()
        need_grad = any(ctx.needs_input_grad)
        z = torch.empty(M, impl.N, dtype=torch.bfloat16, device=x.device) if impl.act != B.ACT_NONE and need_grad else None
        out = impl.forward(x2, bias=bias, z_save=z)
        ctx.layer, ctx.M, ctx.x_shape, ctx.has_bias = layer, M, x.shape, bias is not None
        ctx.save_for_backward(x2, z if z is not None else torch.empty(0, device=x.device))
        return out.reshape(*x.shape[:-1], impl.N)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        layer, M = ctx.layer, ctx.M
        impl = layer.impl
        x2, z = ctx.saved_tensors
        dy2 = dy.reshape(M, impl.N)
        if not dy2.is_contiguous():
            dy2 = dy2.contiguous()
        need_dx = ctx.needs_input_grad[0]
        need_db = ctx.has_bias and ctx.needs_input_grad[2]
        db = torch.empty(impl.N, dtype=torch.float32, device=dy.device) if need_db else None
        dx = impl.backward(dy2, x2, z_saved=z if z.numel() else None, dbias=db, need_dx=need_dx)
        if need_db:
            impl.comm.all_reduce(db, tag="bias")       # the bias is replicated: its gradient is summed over ranks
        # The loop leaves the summed gradients in its own buffers, which the next backward overwrites:
        # autograd gets copies (shard-sized for the ZDP slices, slice-sized for the DP ones).
        g_shard = impl.grad_shard.clone() if ctx.needs_input_grad[1] else None
        g_dp = [impl.dp_grad[s].clone() for s in layer._dp_order]
        return (dx.reshape(ctx.x_shape) if need_dx else None), g_shard, db, None, *g_dp


class ZdpLinear(torch.nn.Module):
    """The split linear layer with its weight sharded over the ranks of a process group, the counterpart of the
    paper's wrapper around a sharded module (Section 3.2, implementation; Section 3.3 for the slices): W is cut
    into `k_split` slices; a ZDP slice is stored as 1 / world of its elements per rank, gathered for use slice by
    slice in forward and backward, and its gradient reduce-scattered; a DP slice (`slice_modes`, e.g. from
    `zdp.slice_modes_from_plan`) is whole on every rank and has its gradient all-reduced.

    Parameters: `shard` (bf16, this rank's part of every ZDP slice), `dp_parts` (the DP slices' compact matrices),
    `bias` (fp32, replicated).  After backward their `.grad` hold this rank's part of the gradient summed over
    ranks (bf16 for the weights, fp32 for the bias), ready for a sharded optimiser step (``optim.ClippedStep`` clips by
    the norm over all ranks, with ``shard`` in a group marked as sharded).  Every rank passes its own tokens.  Collectives run on the layer's communication stream, overlapped with the slice GEMMs.
    """

    def __init__(self, in_features, out_features, bias=True, k_split=1, split_dim=B.SPLIT_OUT, act=B.ACT_NONE,
                 slice_modes=None, comm=None, flags=0, device="cuda"):
        super().__init__()
        from .zdp import ZdpSplitLinear
        self.impl = ZdpSplitLinear(out_features, in_features, k_split, split_dim, act=act, dw_dtype=B.DTYPE_BF16, comm=comm,
                                   device=device, flags=flags, slice_modes=slice_modes)
        self.in_features, self.out_features = int(in_features), int(out_features)
        self.shard = torch.nn.Parameter(self.impl.param_shard)            # same storage: an optimiser step updates the loop's shard
        self._dp_order = sorted(self.impl.dp_weight)
        self.dp_parts = torch.nn.ParameterList([torch.nn.Parameter(self.impl.dp_weight[s]) for s in self._dp_order])
        self.bias = torch.nn.Parameter(torch.zeros(self.out_features, dtype=torch.float32, device=device)) if bias else None

    def load_full_weight(self, w_full):
        """Keeps this rank's part of a full [out_features, in_features] weight."""
        with torch.no_grad():
            self.impl.load_full_weight(w_full)

    def forward(self, x):
        if not x.is_cuda:
            raise RuntimeError("ZdpLinear runs on CUDA only: there is no CPU path")
        if x.dtype != torch.bfloat16:
            raise TypeError("ZdpLinear takes bf16 activations")
        _check_fp32(x.device, bias=(self.bias, self.out_features))
        return _ZdpLinearFn.apply(x, self.shard, self.bias, self, *self.dp_parts)


class _ResidualNormFn(torch.autograd.Function):
    """(r, u) of osdp_block_norm_fwd; r is None where it would be x itself (no y, alpha 1)."""

    @staticmethod
    def forward(ctx, x, y, w_post, b_post, gate, w_pre, b_pre, layer):
        D = layer.hidden
        M = x.numel() // D
        x2 = x.reshape(M, D).contiguous()
        y2 = y.reshape(M, D).contiguous() if y is not None else None
        need_grad = any(ctx.needs_input_grad)
        pre = layer.pre != B.NORM_NONE
        # in the caller's shape: a view made here could not be changed in place under autograd
        r = None if y is None and layer.alpha == 1.0 else torch.empty(x.shape, dtype=x.dtype, device=x.device)
        u = torch.empty(x.shape, dtype=torch.bfloat16, device=x.device) if pre else None
        post = layer.post if y is not None else B.NORM_NONE
        if y is None:
            w_post = b_post = gate = None
        stats = torch.empty(M, 4, dtype=torch.float32, device=x.device) if need_grad else None
        B.osdp_block_norm_fwd(x2, y2, M, D, layer.resid_dtype, post, w_post, b_post, layer.eps, gate, layer.alpha, layer.beta,
                              layer.pre, w_pre, b_pre, layer.eps, r, u, None, stats, check=True)
        if need_grad:
            ctx.layer, ctx.M, ctx.post, ctx.shape = layer, M, post, x.shape
            ctx.save_for_backward(y2, (x2 if r is None else r) if pre else None, stats, w_post, b_post, gate, w_pre)
        ctx.set_materialize_grads(False)
        return r, u

    @staticmethod
    @once_differentiable
    def backward(ctx, dr, du):
        layer, M = ctx.layer, ctx.M
        D = layer.hidden
        y, r, stats, w_post, b_post, gate, w_pre = ctx.saved_tensors
        need = ctx.needs_input_grad
        if dr is None and du is None:
            return (None,) * 8
        dev = stats.device
        pre = layer.pre if du is not None else B.NORM_NONE   # u was not used: nothing comes through its norm
        dr = dr.reshape(M, D).contiguous() if dr is not None else None
        du = du.reshape(M, D).contiguous() if du is not None else None
        has_y = y is not None
        dx = torch.empty(M, D, dtype=layer.resid_torch_dtype, device=dev) if need[0] else None
        dy = torch.empty(M, D, dtype=torch.bfloat16, device=dev) if has_y and need[1] else None
        vec = lambda on: torch.empty(D, dtype=torch.float32, device=dev) if on else None    # noqa: E731
        dw_post, db_post, dgate = vec(need[2] and has_y), vec(need[3] and has_y), vec(need[4] and has_y)
        dw_pre, db_pre = vec(need[5] and pre), vec(need[6] and pre)
        # this call's own: a backward on another stream may run at the same time, a captured one keeps its own
        ws = torch.empty(layer._backward_bytes, dtype=torch.uint8, device=dev)
        B.osdp_block_norm_bwd(dr, du, y, r, stats, M, D, layer.resid_dtype, ctx.post, w_post, b_post, gate, layer.alpha, layer.beta,
                              pre, w_pre if pre else None, dx, dy, dw_post, db_post, dgate, dw_pre, db_pre, ws, check=True)
        return (dx.view(ctx.shape) if dx is not None else None, dy.view(ctx.shape) if dy is not None else None, dw_post, db_post,
                dgate, dw_pre, db_pre, None)


_NORMS = {None: B.NORM_NONE, "rms": B.NORM_RMS, "layer": B.NORM_LAYER}


class ResidualNorm(torch.nn.Module):
    """What stands between two blocks of a transformer, in one kernel:

        r = alpha * x + beta * gate (.) N_post(y),    u = N_pre(r)

    x: the residual stream (bf16, or fp32 with resid_dtype=torch.float32), y: the output of the block before (bf16), r:
    the new residual stream, u (bf16): the input of the block after.  ``forward(x, y)`` returns (r, u);
    ``forward(x)`` in front of the first block leaves the y term out; pre=None returns (r, None) behind the last one.
    post / pre: "rms", "layer" or None.  gate: a learned value per channel (``gate_init``), or none with gate=False.
    Weights, biases and gate are fp32 parameters and have to stay fp32: a module cast by ``to(dtype)`` is refused.

    ``forward_int8(x, y)`` (no gradient) returns (r, (u8, scale)): u as int8 with a scale per token, what ``Int8Linear``
    takes, without the bf16 u in between.
    """

    def __init__(self, hidden, post="rms", pre="rms", gate=True, gate_init=1.0, alpha=1.0, beta=1.0, eps=1e-5,
                 resid_dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        if hidden % 8 or not 0 < hidden <= B.BLOCK_NORM_MAX_D:
            raise ValueError("hidden must be a multiple of 8 and at most %d" % B.BLOCK_NORM_MAX_D)
        if post not in _NORMS or pre not in _NORMS:
            raise ValueError('post and pre are "rms", "layer" or None')
        if resid_dtype not in (torch.bfloat16, torch.float32):
            raise ValueError("the residual stream is bf16 or fp32")
        self.hidden, self.post, self.pre = int(hidden), _NORMS[post], _NORMS[pre]
        self.alpha, self.beta, self.eps = float(alpha), float(beta), float(eps)
        self.resid_torch_dtype = resid_dtype
        self.resid_dtype = B.DTYPE_FP32 if resid_dtype == torch.float32 else B.DTYPE_BF16
        vec = lambda on, v: torch.nn.Parameter(torch.full((self.hidden,), float(v), device=device)) if on else None   # noqa: E731
        self.w_post, self.b_post = vec(post, 1.0), vec(post == "layer", 0.0)
        self.w_pre, self.b_pre = vec(pre, 1.0), vec(pre == "layer", 0.0)
        self.gate = vec(gate, gate_init)
        rc, self._backward_bytes = B.osdp_block_norm_workspace_bytes(0, self.hidden)     # (the same for any number of rows)
        if rc:
            raise B.OsdpError(rc, "osdp_block_norm_workspace_bytes")

    def _check(self, x, y):
        if not x.is_cuda:
            raise RuntimeError("ResidualNorm runs on CUDA only: there is no CPU path")
        if x.dtype != self.resid_torch_dtype or (y is not None and y.dtype != torch.bfloat16):
            raise TypeError("ResidualNorm takes x in its resid_dtype and y in bf16")
        if x.shape[-1] != self.hidden or (y is not None and y.shape != x.shape):
            raise ValueError("x and y are [..., hidden] of the same shape")
        if y is not None and y.device != x.device:
            raise RuntimeError("x is on %s and y on %s: they have to be on one CUDA device" % (x.device, y.device))
        D = self.hidden
        _check_fp32(x.device, w_post=(self.w_post, D), b_post=(self.b_post, D), gate=(self.gate, D), w_pre=(self.w_pre, D), b_pre=(self.b_pre, D))

    def forward(self, x, y=None):
        if _elsewhere(x):
            with torch.cuda.device(x.device):
                return self.forward(x, y)
        self._check(x, y)
        if y is None and self.alpha == 1.0 and self.pre == B.NORM_NONE:
            return x, None
        r, u = _ResidualNormFn.apply(x, y, self.w_post, self.b_post, self.gate, self.w_pre, self.b_pre, self)
        return (x if r is None else r), u

    @torch.no_grad()
    def forward_int8(self, x, y=None):
        if _elsewhere(x):
            with torch.cuda.device(x.device):
                return self.forward_int8(x, y)
        self._check(x, y)
        if self.pre == B.NORM_NONE:
            raise ValueError("there is no u to quantise: pre is None")
        D = self.hidden
        M = x.numel() // D
        x2 = x.reshape(M, D).contiguous()
        y2 = y.reshape(M, D).contiguous() if y is not None else None
        r = None if y is None and self.alpha == 1.0 else torch.empty_like(x2)      # (x itself, as in forward)
        u = torch.empty(M, D, dtype=torch.int8, device=x.device)
        s = torch.empty(M, dtype=torch.float32, device=x.device)
        post, w_post, b_post, gate = (self.post, self.w_post, self.b_post, self.gate) if y is not None else (B.NORM_NONE, None, None, None)
        B.osdp_block_norm_fwd(x2, y2, M, D, self.resid_dtype, post, w_post, b_post, self.eps, gate, self.alpha, self.beta, self.pre,
                              self.w_pre, self.b_pre, self.eps, r, u, s, None, check=True)
        return (x if r is None else r.view(x.shape)), (u.view(x.shape), s.view(x.shape[:-1]))


def quantize_int8(x):
    """(int8 rows, fp32 scale per row) of a bf16 tensor [..., K] (osdp_quantize_rows_i8)."""
    K = x.shape[-1]
    if not x.is_cuda or x.dtype != torch.bfloat16:
        raise TypeError("quantize_int8 takes a bf16 CUDA tensor")
    if _elsewhere(x):
        with torch.cuda.device(x.device):
            return quantize_int8(x)
    x2 = x.detach().reshape(-1, K).contiguous()
    q = torch.empty(x2.shape, dtype=torch.int8, device=x.device)
    s = torch.empty(x2.shape[0], dtype=torch.float32, device=x.device)
    B.osdp_quantize_rows_i8(x2, x2.shape[0], K, q, s, check=True)
    return q.view(x.shape), s.view(x.shape[:-1])


class _Int8LinearFn(torch.autograd.Function):
    """Int8Linear on an input that has a gradient: says so when that is asked for, instead of cutting the graph."""

    @staticmethod
    def forward(ctx, x, layer):
        return layer._product(x, None)

    @staticmethod
    def backward(ctx, dy):
        raise RuntimeError("Int8Linear has no gradient: train the layer it was made from")


class Int8Linear(torch.nn.Module):
    """y = act(x W^T + b) for serving, with int8 weights (a scale per output channel) and int8 activations (a scale per
    token, taken from the token itself); int32 sums, bf16 output.  No gradient: a backward pass through it raises.

    weight8 [out, in] int8, w_scale [out] fp32, bias [out] fp32 or None (fp32 for good: a module cast by ``to(dtype)`` is
    refused).  ``from_linear`` quantises a trained
    ``SplitLinear`` (or any bf16 weight).  ``forward`` takes bf16 activations, or the pair (int8, scale) that
    ``ResidualNorm.forward_int8`` and ``quantize_int8`` return.
    Nothing of a call is kept: calls on several streams and replays of captured graphs do not meet.
    """

    def __init__(self, weight8, w_scale, bias=None, act=B.ACT_NONE, k_split=1, split_dim=B.SPLIT_OUT):
        super().__init__()
        if weight8.dtype != torch.int8 or weight8.dim() != 2 or w_scale.dtype != torch.float32 or w_scale.numel() != weight8.shape[0]:
            raise ValueError("weight8 is [out, in] int8 with one fp32 scale per row")
        if bias is not None and (bias.dtype != torch.float32 or bias.numel() != weight8.shape[0]):
            raise ValueError("bias is [out] fp32")
        self.out_features, self.in_features = weight8.shape
        if self.in_features % 16 or self.out_features % 8:
            raise ValueError("in_features must be a multiple of 16 and out_features of 8")
        self.register_buffer("weight8", weight8.contiguous())
        self.register_buffer("w_scale", w_scale.contiguous())
        self.register_buffer("bias", bias.contiguous() if bias is not None else None)
        self.act, self.k_split, self.split_dim = int(act), int(k_split), int(split_dim)
        # the tile kernel's status word: all that is kept between calls
        self.register_buffer("_status", torch.zeros(256, dtype=torch.uint8, device=weight8.device), persistent=False)

    @classmethod
    def from_linear(cls, layer, **kw):
        """From a SplitLinear, or from anything with a bf16 `weight` [out, in] and an optional `bias`."""
        q, s = quantize_int8(layer.weight)
        bias = layer.bias.detach().float() if layer.bias is not None else None
        return cls(q, s, bias, act=getattr(layer, "act", B.ACT_NONE), **kw)

    def forward(self, x):
        q, s = x if isinstance(x, tuple) else (x, None)
        if q.dtype != (torch.bfloat16 if s is None else torch.int8) or not q.is_cuda:
            raise TypeError("Int8Linear takes bf16 CUDA activations, or a pair (int8, fp32 scale per token)")
        if _elsewhere(q):
            with torch.cuda.device(q.device):
                return self.forward(x)
        if q.requires_grad and torch.is_grad_enabled():
            return _Int8LinearFn.apply(q, self)
        return self._product(q, s)

    def _check(self, q, w8, w_scale, bias):
        if w8.dtype is not torch.int8 or w8.device != q.device or w8.numel() != self.out_features * self.in_features or not w8.is_contiguous():
            raise RuntimeError("weight8 has to be contiguous [out_features, in_features] int8 on %s, its input's device" % q.device)
        _check_fp32(q.device, w_scale=(w_scale, self.out_features), bias=(bias, self.out_features))

    def _product(self, q, s):
        K, N = self.in_features, self.out_features
        shape = q.shape
        if shape[-1] != K:
            raise ValueError("Int8Linear takes [..., in_features]")
        M = q.numel() // K
        held = self._buffers          # (an attribute of a module that is a buffer takes several times as long)
        w8, w_scale, bias, device = held["weight8"], held["w_scale"], held["bias"], q.device
        if w8.dtype is not torch.int8 or w8.device != device or w8.numel() != N * K or not w8.is_contiguous() or \
           w_scale.dtype is not torch.float32 or w_scale.device != device or w_scale.numel() != N or not w_scale.is_contiguous() or \
           (bias is not None and (bias.dtype is not torch.float32 or bias.device != device or bias.numel() != N or not bias.is_contiguous())):
            self._check(q, w8, w_scale, bias)
        if not q.is_contiguous():
            q = q.contiguous()
        stream = B._stream(None)
        if s is not None:
            if s.dtype != torch.float32 or s.numel() != M:
                raise ValueError("one fp32 scale per token")
            if s.device != device:
                raise RuntimeError("the scales are on %s and the tokens on %s: they have to be on one CUDA device" % (s.device, device))
            s = s.contiguous()
        else:
            # This call's own scales (whole 256-byte lines of them) and codes: another stream's call has others, and a
            # captured graph keeps its own.
            lines = -(-M // 64) * 256
            own = torch.empty(lines + M * K, dtype=torch.uint8, device=device)
            s = own.data_ptr()
            B.osdp_quantize_rows_i8(q, M, K, s + lines, s, stream, True)
            q = s + lines
        out = torch.empty(shape[:-1] + (N,), dtype=torch.bfloat16, device=device)
        B.osdp_split_linear_fwd_i8(q, s, w8, 0, w_scale, bias, M, N, K, self.k_split, self.split_dim, self.act, out, held["_status"], stream,
                                   True)
        return out
