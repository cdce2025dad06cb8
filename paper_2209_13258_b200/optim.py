"""AdamW over the parameters of the split layers: one kernel launch for all tensors, states in 32 or in 8 bits, and the
gradient norm with its clipping coefficient on the device.

Argument marshalling only; the arithmetic runs in ``osdp_adamw_step`` / ``osdp_grad_norm``.  CUDA only.
"""
from __future__ import annotations

import operator

import numpy as np
import torch

from . import binding as B

_TENSOR = np.dtype([("param", np.uint64), ("grad", np.uint64), ("numel", np.int64), ("state_offset", np.int64),
                    ("lr", np.float64), ("weight_decay", np.float64)])      # osdp_adamw_tensor


_STATES = {"fp32": B.DTYPE_FP32, "e4m3": B.DTYPE_E4M3, "e4m3_dithered": B.DTYPE_E4M3_DITHERED}
_GRAD, _DTYPE, _VERSION = operator.attrgetter("grad"), operator.attrgetter("dtype"), operator.attrgetter("_version")
_DATA_PTR, _NUMEL, _DEVICE, _IS_CONTIGUOUS = torch.Tensor.data_ptr, torch.Tensor.numel, torch.Tensor.get_device, torch.Tensor.is_contiguous


try:      # what torch's wrapper around an optimiser's step looks at: without a hook or a profiler it has nothing to do
    from torch.autograd import _profiler_enabled
    from torch.optim.optimizer import _global_optimizer_post_hooks, _global_optimizer_pre_hooks
except ImportError:
    _profiler_enabled, _global_optimizer_post_hooks, _global_optimizer_pre_hooks = (lambda: True), {}, {}
try:      # one native pass over type, dtype, device, sizes and strides of many tensors, where this torch has it
    from torch._C._dynamo.guards import TensorGuards as _TensorGuards
except ImportError:
    _TensorGuards = None


def _guard_of(tensors):
    return _TensorGuards(*tensors, dynamic_dims_sizes=[list(t.shape) for t in tensors], dynamic_dims_strides=[list(t.stride()) for t in tensors])


class AdamW(torch.optim.Optimizer):
    """Decoupled weight decay (AdamW) for contiguous CUDA parameters of one dtype, bf16 or fp32.

    state_dtype  "fp32", or "e4m3": both moments as 8-bit codes with one fp32 scale per 256 elements (2.03 bytes per
                 parameter instead of 8; the second moment is kept as its root).
                 A moment whose beta is at most 0.975 is rounded to the nearest code, others up or down at random
                 (repeatably: by element and step), since the nearest code would hold them where they are.  "e4m3_dithered":
                 at random whatever the betas, for gradients with next to no noise of their own.
    master       bf16 parameters only: the step works on fp32 copies of the parameters (4 bytes each) and writes their
                 rounding.  Without it an update below half a unit in the last place of a bf16 parameter is lost.
                 Parameters that change outside the step (weights loaded, averaged or initialised again: any in-place
                 operation on them, or new ``.data``) are noticed by the next step, which takes the changed elements over
                 into the masters.  Writes through ``p.data`` or by another library's kernels leave no trace:
                 call ``refresh_masters()`` after them.
    max_norm     clips the gradients by their norm over all parameters of the step, without a host round trip.  That is
                 this optimiser's norm on this rank: parameters of two dtypes, or sharded over ranks, have to be clipped
                 together, or their parts are scaled differently (and replicated parameters drift apart): ``ClippedStep``.
                 A step whose norm is not finite changes no parameter and no state (``grad_norm[0]`` says so); it counts as
                 a step all the same, since the host does not wait to learn of it.

    All parameter groups are stepped together: ``lr`` and ``weight_decay`` may differ between groups, ``betas`` and
    ``eps`` may not.  A group with ``"sharded": True`` says that every rank has other elements of its parameters.
    Parameters whose ``.grad`` is None are left alone.  ``steps`` counts the steps done (one count for all parameters: it
    sets the bias correction).  States are flat over all parameters, each parameter's part starting
    at a multiple of 256 elements (``offsets``): ``exp_avg``, ``exp_avg_sq`` (in 8 bits the codes of the second
    moment's root), ``exp_avg_scale``, ``exp_avg_sq_scale``, ``master``.  A CUDA graph of a step replays that step's
    bias correction, rates and gradients' addresses.  ``grad_norm`` [2]: the last step's norm and
    coefficient, on the device.
    """

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, state_dtype="fp32", master=False,
                 max_norm=None):
        if state_dtype not in _STATES:
            raise ValueError('state_dtype is "fp32", "e4m3" or "e4m3_dithered"')
        self._built = False
        super().__init__(params, {"lr": lr, "betas": tuple(betas), "eps": eps, "weight_decay": weight_decay})
        self._params = [p for g in self.param_groups for p in g["params"]]
        first = self._params[0]
        if first.dtype not in (torch.bfloat16, torch.float32):
            raise TypeError("AdamW takes bf16 or fp32 parameters")
        for p in self._params:
            if not p.is_cuda:
                raise RuntimeError("AdamW runs on CUDA only: there is no CPU path")
            if p.dtype != first.dtype or p.device != first.device:
                raise TypeError("the parameters of one AdamW have one dtype and one device")
            if not p.is_contiguous():
                raise ValueError("AdamW takes contiguous parameters")
        if master and first.dtype != torch.bfloat16:
            raise ValueError("fp32 parameters are their own master")
        self._torch_dtype, self._device = first.dtype, first.device
        self._dtype = B.DTYPE_FP32 if first.dtype == torch.float32 else B.DTYPE_BF16
        self._state_dtype = _STATES[state_dtype]
        eight = state_dtype != "fp32"
        rc, self.offsets, total = B.osdp_adamw_layout([p.numel() for p in self._params])
        if rc:
            raise B.OsdpError(rc, "osdp_adamw_layout")
        dev = first.device
        new = lambda n, dt: torch.zeros(n, dtype=dt, device=dev)      # noqa: E731
        sdt = torch.float8_e4m3fn if eight else torch.float32
        self.exp_avg, self.exp_avg_sq = new(total, sdt), new(total, sdt)
        blocks = total // B.ADAMW_BLOCK
        self.exp_avg_scale, self.exp_avg_sq_scale = (new(blocks, torch.float32), new(blocks, torch.float32)) if eight else (None, None)
        self.master = None
        if master:
            self.master = new(total, torch.float32)
            for p, o in zip(self._params, self.offsets):
                self.master[o:o + p.numel()].copy_(p.detach().reshape(-1))
        self._seen = self._params_now() if master else None
        self.max_norm = max_norm
        self.grad_norm = new(2, torch.float32)
        self.steps = 0
        n = len(self._params)
        # the step's table of tensors, filled column by column; `_whole`: its sizes, offsets and rates are those of all
        # parameters in order
        self._sizes = [p.numel() for p in self._params]
        self._group_of = [i for i, g in enumerate(self.param_groups) for _ in g["params"]]
        self.sharded = np.array([bool(g.get("sharded", False)) for g in self.param_groups for _ in g["params"]])
        if max_norm is not None and self.sharded.any():
            raise ValueError("sharded parameters are clipped by the norm over all ranks: ClippedStep")
        self._clip = None       # coefficient from outside, while a ClippedStep steps
        self._table = np.zeros(n, dtype=_TENSOR)
        self._table_at = self._table.ctypes.data
        self._whole, self._rates = False, None
        self._written = None, None      # the addresses that the table's first entries hold
        # parameters and gradients as one step found them in order; a few times anew, if what comes changes
        self._guard, self._guards_left = None, 9 if _TensorGuards is not None else 0
        self._ws = B.new_workspace(B.osdp_grad_norm_workspace_bytes(n)[1], device=dev)
        self._built = True

    def add_param_group(self, group):
        if self._built:
            raise RuntimeError("the states are laid out when the optimiser is built: pass all groups then")
        super().add_param_group(group)

    def _params_now(self):
        """Changes with every in-place operation on a parameter (the step's own kernel leaves it alone) and every move."""
        return list(map(_VERSION, self._params)), list(map(_DATA_PTR, self._params))

    @torch.no_grad()
    def refresh_masters(self):
        """Takes parameters over into the fp32 masters, element by element where a parameter is not its master's
        rounding: elements that nobody changed keep their masters' digits."""
        if self.master is None:
            return
        for p, o, n in zip(self._params, self.offsets, self._sizes):
            m, w = self.master[o:o + n], p.detach().reshape(-1)
            m.copy_(torch.where(m.to(w.dtype) == w, m, w.to(m.dtype)))
        self._seen = self._params_now()

    def _refuse(self, what, tensors, sizes):
        """Raises for the tensor that is no longer what the kernel is told of it."""
        for i, (t, n) in enumerate(zip(tensors, sizes)):
            if t.dtype is not self._torch_dtype:
                raise TypeError("%s %d is %s, the optimiser was built for %s" % (what, i, t.dtype, self._torch_dtype))
            if t.get_device() != self._device.index:
                raise RuntimeError("%s %d is on %s, the optimiser was built on %s" % (what, i, t.device, self._device))
            if t.numel() != n:
                raise ValueError("%s %d has %d elements, the optimiser was built for %d" % (what, i, t.numel(), n))
            if what == "parameter" and not t.is_contiguous():
                raise ValueError("parameter %d is not contiguous any more" % i)

    def _fill(self):
        """The table of this step: addresses as they are now; tensors without a gradient are left out.  Returns its
        length, the copies of gradients that were not contiguous, and the indices of its parameters (None: all)."""
        params, table, sizes = self._params, self._table, self._sizes
        grads, at, keep = list(map(_GRAD, params)), None, None
        # The kernel has addresses and the lengths recorded when the optimiser was built: whatever else a parameter or a
        # gradient has become (moved, cast, resized, strided) would be read and written out of its bounds.
        if self._guard is None or not self._guard.check(*params, *grads):
            if type(None) in set(map(type, grads)):
                at = [i for i, g in enumerate(grads) if g is not None]
            dtype, device = {self._torch_dtype}, {self._device.index}
            if set(map(_DTYPE, params)) != dtype or set(map(_DEVICE, params)) != device or list(map(_NUMEL, params)) != sizes or \
               not all(map(_IS_CONTIGUOUS, params)):
                self._refuse("parameter", params, sizes)
            if at is not None:
                params, grads, sizes = [params[i] for i in at], [grads[i] for i in at], [sizes[i] for i in at]
            if grads and (set(map(_DTYPE, grads)) != dtype or set(map(_DEVICE, grads)) != device or list(map(_NUMEL, grads)) != sizes):
                self._refuse("gradient", grads, sizes)
            if not all(map(_IS_CONTIGUOUS, grads)):
                keep = grads = [g.contiguous() for g in grads]
            elif at is None and self._guards_left:
                self._guards_left -= 1
                if self._guards_left < 8:       # (not in the first step, which is long enough)
                    self._guard = _guard_of(params + grads)
        n = len(grads)
        rates = [(float(g["lr"]), float(g["weight_decay"])) for g in self.param_groups]
        if at is not None or not self._whole or rates != self._rates:
            which = range(n) if at is None else at
            table["numel"][:n] = [self._sizes[i] for i in which]
            table["state_offset"][:n] = [self.offsets[i] for i in which]
            table["lr"][:n] = [rates[self._group_of[i]][0] for i in which]
            table["weight_decay"][:n] = [rates[self._group_of[i]][1] for i in which]
            self._whole, self._rates = at is None, rates
        at_params, at_grads = list(map(_DATA_PTR, params)), list(map(_DATA_PTR, grads))
        if at_params != self._written[0]:      # (comparing lists takes a tenth of writing a column)
            table["param"][:n] = at_params
        if at_grads != self._written[1]:
            table["grad"][:n] = at_grads
        self._written = at_params, at_grads
        return n, keep, at

    def _step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        first = self.param_groups[0]
        betas, eps = first["betas"], first["eps"]
        for g in self.param_groups:
            if g["betas"] != betas or g["eps"] != eps:
                raise ValueError("betas and eps are the same for all groups")
        if torch.cuda.current_device() != self._device.index:
            with torch.cuda.device(self._device):
                self._launch(betas, eps)
        else:
            self._launch(betas, eps)
        return loss

    _wrapped_step = torch.optim.Optimizer.profile_hook_step(_step)

    def step(self, *args, **kwargs):
        """step(closure=None): one step; returns the closure's loss."""
        if self._optimizer_step_pre_hooks or self._optimizer_step_post_hooks or _global_optimizer_pre_hooks or \
           _global_optimizer_post_hooks or _profiler_enabled():
            return self._wrapped_step(*args, **kwargs)
        return self._step(*args, **kwargs)

    step.hooked = True       # torch's wrapper is called here, where it has something to do: its profiler range alone takes 13 us

    def _launch(self, betas, eps):
        n, keep, _ = self._fill()
        if self.master is not None and self._params_now() != self._seen:
            self.refresh_masters()
        step = self.steps + 1
        clip, table = self._clip, self._table_at
        if clip is None and self.max_norm is not None:
            clip = self.grad_norm
            B.osdp_grad_norm(table, n, self._dtype, self.max_norm, clip, self._ws, check=True)
        B.osdp_adamw_step(table, n, self._dtype, self._state_dtype, self.master, self.exp_avg, self.exp_avg_sq, self.exp_avg_scale,
                          self.exp_avg_sq_scale, betas[0], betas[1], eps, step, clip, check=True)
        self.steps = step        # (not of a step that was refused)

    def _squares(self, replicated, sharded):
        """Sums of squares of the gradients of replicated and of sharded parameters into two fp64 values on the device
        (None: that part is not wanted)."""
        n, keep, at = self._fill()
        flags = self.sharded if at is None else self.sharded[at]
        for to, which in ((replicated, ~flags), (sharded, flags)):
            if to is not None:
                part = np.ascontiguousarray(self._table[:n][which])
                B.osdp_grad_squares(part.ctypes.data, len(part), self._dtype, to, self._ws, check=True)

    def __getstate__(self):
        raise TypeError("an AdamW is copied or saved through state_dict()")     # torch's copy would leave the flat states out

    def state_dict(self):
        d = super().state_dict()
        d["flat"] = {k: getattr(self, k) for k in ("exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale", "master")}
        d["steps"] = self.steps
        return d

    def load_state_dict(self, d):
        d = dict(d)
        flat, steps = d.pop("flat"), d.pop("steps")
        for k, v in flat.items():
            mine = getattr(self, k)
            if (mine is None) != (v is None) or (v is not None and (mine.shape != v.shape or mine.dtype != v.dtype)):
                raise ValueError("%s does not fit this optimiser" % k)
        super().load_state_dict(d)
        for k, v in flat.items():
            if v is not None:
                getattr(self, k).copy_(v)
        self.steps = int(steps)
        if self.master is not None:
            self._seen = self._params_now()


class ClippedStep:
    """Steps several ``AdamW`` optimisers with their gradients clipped by ONE norm: over all their parameters, whatever their
    dtypes, and over the ranks of a process group.

        opt = ClippedStep([AdamW(bf16_params, ...), AdamW(fp32_params, ...)], max_norm=1.0)
        loss.backward(); opt.step(); opt.zero_grad()

    comm      rank, world and all_reduce(tensor) of the ranks (``zdp.DistComm``), or None: one process.  Parameters in groups
              with ``"sharded": True`` (``ZdpLinear.shard``) have other elements on every rank: their sums of squares are
              added over ranks.  All others are replicated with the same gradients everywhere (``ZdpLinear.dp_parts``,
              biases): rank 0's are counted.  So every rank has the same coefficient, bit by bit.  Every rank calls
              ``step()``: it is a collective.
    max_norm  as in AdamW; the optimisers themselves have none.  A norm that is not finite changes nothing on any rank.

    ``grad_norm`` [2]: the last step's norm and coefficient, on the device.  The norm is taken before the optimisers' own
    hooks run.
    """

    def __init__(self, optimizers, max_norm, comm=None):
        self.optimizers, self.max_norm, self.comm = list(optimizers), float(max_norm), comm
        if not self.optimizers or not all(isinstance(o, AdamW) for o in self.optimizers):
            raise TypeError("ClippedStep takes AdamW optimisers")
        if any(o.max_norm is not None for o in self.optimizers):
            raise ValueError("the optimisers of a ClippedStep have no max_norm of their own")
        self._device = self.optimizers[0]._device
        if any(o._device != self._device for o in self.optimizers):
            raise RuntimeError("the optimisers of a ClippedStep are on one device")
        if comm is None and any(o.sharded.any() for o in self.optimizers):
            raise ValueError("sharded parameters are clipped over the ranks of a comm")
        self.grad_norm = torch.zeros(2, dtype=torch.float32, device=self._device)
        self._sums = torch.zeros(2 * len(self.optimizers), dtype=torch.float64, device=self._device)

    def _local_sums(self):
        """This rank's sums of squares: of what is replicated (rank 0 alone, zeros elsewhere), then of what is sharded."""
        k, at = len(self.optimizers), self._sums.data_ptr()
        first = self.comm is None or self.comm.rank == 0
        if not first:
            self._sums.zero_()      # the last all-reduce's results
        for i, o in enumerate(self.optimizers):
            o._squares(at + 8 * i if first else None, at + 8 * (k + i) if self.comm is not None else None)
        return self._sums

    @torch.no_grad()
    def step(self):
        with torch.cuda.device(self._device):
            sums = self._local_sums()
            if self.comm is not None:
                self.comm.all_reduce(sums, tag="grad_norm")
            B.osdp_clip_coefficient(sums, sums.numel() if self.comm is not None else len(self.optimizers), self.max_norm, self.grad_norm, check=True)
            for o in self.optimizers:
                o._clip = self.grad_norm
                try:
                    o.step()
                finally:
                    o._clip = None

    def zero_grad(self, set_to_none=True):
        for o in self.optimizers:
            o.zero_grad(set_to_none=set_to_none)
