"""Workloads of the operators around the split linear layers: the norms, gate and residual sum between two blocks
(forward and backward), the AdamW step over the flat parameters, and the int8 linear layer of the serving path.

`run` computes them in elementary torch operations in 32 bits, or, with `own` set, with this package's kernels.
"""
import math
import random

import torch

own = False

QB = 256            # elements that share one scale of an 8-bit optimiser state
TINY = 2.0 ** -100  # a block of 256 whose largest magnitude is below this is stored as zeros
F32, BF16, F8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


def listed():
    return [
        # --- AdamW ---
        # the parameters of one small MLP block (hidden 512): a step whose cost is its launches
        {"name": "adamw-block-512", "op": "adamw", "hidden": 512, "ffn": 2048, "layers": 1, "param": "bf16", "master": True,
         "state": "fp32", "clip": False},
        # four MLP blocks of a hidden-2048 model, bf16 parameters with fp32 masters, gradients clipped by their norm
        {"name": "adamw-4x2048-clip", "op": "adamw", "hidden": 2048, "ffn": 8192, "layers": 4, "param": "bf16", "master": True,
         "state": "fp32", "clip": True},
        # a shard that holds pieces of many tensors, none of a round size: fp32 parameters, 8-bit states
        {"name": "adamw8-ragged", "op": "adamw", "tensors": 173, "total": 21_000_001, "mix": 5, "param": "fp32", "master": False,
         "state": "e4m3", "clip": True},
        # the wide block (hidden 8192, ffn 32768): bf16 parameters, 8-bit states, no master: the memory-saving setting
        {"name": "adamw8-wide", "op": "adamw", "hidden": 8192, "ffn": 32768, "layers": 1, "param": "bf16", "master": False,
         "state": "e4m3", "clip": False},
        # --- norms, gate and residual sum ---
        # one token between two blocks while a sequence is generated
        {"name": "norm-fwd-token", "op": "norm", "dir": "fwd", "M": 1, "D": 2048, "kind": "rms", "resid": "bf16", "gate": True},
        # a training batch of the hidden-2048 model, layer norms, fp32 residual stream
        {"name": "norm-fwd-2048", "op": "norm", "dir": "fwd", "M": 8192, "D": 2048, "kind": "layer", "resid": "fp32", "gate": True},
        # a ragged batch of a narrow model, backward
        {"name": "norm-bwd-ragged", "op": "norm", "dir": "bwd", "M": 1777, "D": 1032, "kind": "layer", "resid": "bf16", "gate": True},
        # the wide model's training batch, forward and backward
        {"name": "norm-fwd-8192", "op": "norm", "dir": "fwd", "M": 16384, "D": 8192, "kind": "rms", "resid": "bf16", "gate": True},
        {"name": "norm-bwd-8192", "op": "norm", "dir": "bwd", "M": 16384, "D": 8192, "kind": "rms", "resid": "bf16", "gate": True},
        # --- int8 linear layer ---
        # one token through a square layer: reading the weights once is the whole cost
        {"name": "i8-token", "op": "i8", "M": 1, "N": 8192, "K": 8192, "act": False, "bias": True},
        # a handful of sequences, odd batch, first layer of the MLP with its GeLU
        {"name": "i8-batch-37", "op": "i8", "M": 37, "N": 8200, "K": 2064, "act": True, "bias": True},
        # a prompt batch through the wide first layer
        {"name": "i8-prompt", "op": "i8", "M": 8192, "N": 32768, "K": 8192, "act": True, "bias": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _extent(rng, lo, hi, step):
    """A multiple of `step` in [lo, hi], spread over the logarithm."""
    n = max(lo // step, min(hi // step, round(_log(rng, lo, hi) / step))) * step
    return n + step if n == 3072 else n


def draw(rng):
    op = rng.choice(["adamw", "norm", "i8"])
    if op == "adamw":
        param, state = rng.choice(["bf16", "fp32"]), rng.choice(["fp32", "e4m3"])
        n = _log(rng, 1, 400)
        return {"op": op, "tensors": n, "total": max(2 * n, _log(rng, 5000, 130_000_000)), "mix": rng.randrange(1000), "param": param,
                "master": param == "bf16" and state == "fp32" and rng.random() < 0.7, "state": state, "clip": rng.random() < 0.5}
    if op == "norm":
        D = _extent(rng, 64, 16384, 8)
        top = max(2, min(16384, (16384 * 8192) // D // 2))
        return {"op": op, "dir": rng.choice(["fwd", "bwd"]), "M": _log(rng, 1, top), "D": D, "kind": rng.choice(["rms", "layer"]),
                "resid": rng.choice(["bf16", "fp32"]), "gate": rng.random() < 0.7}
    M = _log(rng, 1, 8192)
    M = M + 1 if M == 3072 else M
    return {"op": op, "M": M, "N": _extent(rng, 64, 16384, 8), "K": _extent(rng, 64, 16384, 16), "act": rng.random() < 0.5,
            "bias": rng.random() < 0.7}


# ---------------------------------------------------------------------------------------------------------------------
# inputs

def _gen(seed, dev="cuda"):
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    return g


def _dtype(name):
    return {"bf16": BF16, "fp32": F32}[name]


def _sizes(case):
    """Elements of every parameter tensor, and how many of the tensors (the first ones) have weight decay."""
    if "hidden" in case:
        h, f, n = case["hidden"], case["ffn"], case["layers"]
        return [h * f] * (2 * n) + [f, h, h, h] * n, 2 * n      # w1, w2 of every block; then b1, b2, norm weight, gate
    n, total = case["tensors"], case["total"]
    r = random.Random(case["mix"])
    share = [math.exp(r.uniform(0.0, 5.0)) for _ in range(n)]
    sizes = [max(1, int(total * s / sum(share))) for s in share]
    return sizes, (3 * n + 3) // 4


def _offsets(sizes):
    """Where each tensor starts in the flat buffers (multiples of 256 elements), and the buffers' length."""
    starts, at = [], 0
    for n in sizes:
        starts.append(at)
        at += -(-n // QB) * QB
    return starts, at


HYPER = {"lr": 1e-4, "b1": 0.9, "b2": 0.95, "eps": 1e-8, "wd": 0.1, "max_norm": 1.0, "step": 40}


def _quantise(x, root):
    """Flat fp32 -> e4m3 codes and one scale per 256 elements: scale = max / 448."""
    b = x.view(-1, QB)
    top = b.abs().amax(1)
    live = top >= TINY
    inv = torch.where(live, 448.0 / top, torch.zeros_like(top))
    c = b * inv[:, None]
    if root:   # a root above zero never becomes zero: it would turn a small second moment into a huge step
        c = torch.where((b > 0) & live[:, None], c.clamp_min(2.0 ** -9), c)
    return c.to(F8).view(-1), torch.where(live, top * (1.0 / 448.0), torch.zeros_like(top))


def _inputs(case, seed):
    """What both forms start from."""
    g = _gen(seed)
    if case["op"] == "adamw":
        sizes, n_decay = _sizes(case)
        starts, total = _offsets(sizes)
        keep = torch.zeros(total, dtype=torch.bool, device="cuda")
        for o, n in zip(starts, sizes):
            keep[o:o + n] = True
        rnd = lambda std: torch.randn(total, device="cuda", generator=g).mul_(std).mul_(keep)      # noqa: E731
        p = rnd(0.02)
        param = p.to(_dtype(case["param"]))
        scale = torch.exp(torch.randn(total // QB, 1, device="cuda", generator=g)).mul_(3e-4)      # gradient sizes differ by tensor part
        grad = (rnd(1.0).view(-1, QB) * scale).view(-1).to(_dtype(case["param"]))
        m = (rnd(0.3).view(-1, QB) * scale).view(-1)
        v = ((rnd(1.0).abs_() * 0.5 + 0.75).view(-1, QB) * scale).view(-1).square_().mul_(keep)
        s = {"sizes": sizes, "starts": starts, "n_decay": n_decay, "param": param, "grad": grad, "steps": HYPER["step"],
             "cut": starts[n_decay] if n_decay < len(sizes) else total}
        s["master"] = (p if case["master"] else None)
        if case["state"] == "e4m3":
            s["m"], s["sm"] = _quantise(m, False)
            s["v"], s["sv"] = _quantise(v.sqrt_(), True)
        else:
            s["m"], s["v"] = m, v
        return s
    if case["op"] == "norm":
        M, D = case["M"], case["D"]
        rd, layer = _dtype(case["resid"]), case["kind"] == "layer"
        rnd = lambda *n: torch.randn(*n, device="cuda", generator=g)                                # noqa: E731
        s = {"y": (rnd(M, D) * 0.7 + 0.2 * rnd(D)).to(BF16), "w_post": 1.0 + 0.2 * rnd(D), "w_pre": 1.0 + 0.2 * rnd(D),
             "b_post": 0.1 * rnd(D) if layer else None, "b_pre": 0.1 * rnd(D) if layer else None,
             "gate": 0.5 + 0.2 * rnd(D) if case["gate"] else None, "eps": 1e-5, "alpha": 1.0, "beta": 0.7, "layer": layer,
             "M": M, "D": D}
        stream = (rnd(M, D) * (0.5 + rnd(D).abs()) + 0.3 * rnd(D)).to(rd)
        if case["dir"] == "fwd":
            s["x"] = stream
            return s
        s["r"] = stream
        s["dr"], s["du"] = (rnd(M, D) * 0.1).to(rd), (rnd(M, D) * 0.1).to(BF16)
        s["stats"] = torch.cat([_statistics(s["y"].float(), layer, s["eps"]), _statistics(stream.float(), layer, s["eps"])], 1)
        return s
    M, N, K = case["M"], case["N"], case["K"]
    w = torch.randn(N, K, device="cuda", generator=g).mul_(0.02)
    ws = w.abs().amax(1).clamp_min(1e-20) / 127.0
    wq = torch.round(w.div_(ws[:, None])).to(torch.int8)
    del w
    loud = torch.where(torch.rand(K, device="cuda", generator=g) < 0.01, 8.0, 1.0)                 # a few outlier channels
    return {"x": (torch.randn(M, K, device="cuda", generator=g) * loud).to(BF16), "wq": wq, "ws": ws,
            "bias": torch.randn(N, device="cuda", generator=g) * 0.1 if case["bias"] else None, "act": case["act"]}


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if not own:
        return s
    # what a program keeps between calls: the optimiser, the layer, output buffers and workspace
    import paper_2209_13258_b200 as P
    if case["op"] == "adamw":
        from paper_2209_13258_b200.optim import AdamW
        leaves = [torch.nn.Parameter(s["param"][o:o + n]) for o, n in zip(s["starts"], s["sizes"])]
        for p, o, n in zip(leaves, s["starts"], s["sizes"]):
            p.grad = s["grad"][o:o + n]
        k = s["n_decay"]
        groups = [{"params": leaves[:k], "weight_decay": HYPER["wd"]}]
        if k < len(leaves):
            groups.append({"params": leaves[k:], "weight_decay": 0.0})
        opt = AdamW(groups, lr=HYPER["lr"], betas=(HYPER["b1"], HYPER["b2"]), eps=HYPER["eps"], state_dtype=case["state"],
                    master=case["master"], max_norm=HYPER["max_norm"] if case["clip"] else None)
        opt.steps = s["steps"]
        opt.exp_avg.copy_(s["m"])
        opt.exp_avg_sq.copy_(s["v"])
        if case["state"] == "e4m3":
            opt.exp_avg_scale.copy_(s["sm"])
            opt.exp_avg_sq_scale.copy_(s["sv"])
        if case["master"]:
            opt.master.copy_(s["master"])
        del s["m"], s["v"], s["master"]
        s["opt"] = opt
    elif case["op"] == "norm":
        M, D, rd = s["M"], s["D"], _dtype(case["resid"])
        new = lambda dt, *n: torch.empty(*n, dtype=dt, device="cuda")                               # noqa: E731
        if case["dir"] == "fwd":
            s["out"] = (new(rd, M, D), new(BF16, M, D), new(F32, M, 4))
        else:
            s["out"] = {"dx": new(rd, M, D), "dy": new(BF16, M, D), "dw_post": new(F32, D), "dw_pre": new(F32, D)}
            if s["layer"]:
                s["out"] |= {"db_post": new(F32, D), "db_pre": new(F32, D)}
            if s["gate"] is not None:
                s["out"]["dgate"] = new(F32, D)
            s["ws"] = P.new_workspace(P.osdp_block_norm_workspace_bytes(M, D)[1])
    else:
        from paper_2209_13258_b200.nn import Int8Linear
        s["layer"] = Int8Linear(s["wq"], s["ws"], s["bias"], act=P.ACT_GELU_TANH if s["act"] else P.ACT_NONE)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# the framework's calls

def _run_own(s):
    import paper_2209_13258_b200 as P
    case = s["case"]
    if case["op"] == "adamw":
        opt = s["opt"]
        opt.step()
        out = {"param": s["param"], "m": opt.exp_avg, "v": opt.exp_avg_sq}
        if case["master"]:
            out["master"] = opt.master
        if case["state"] == "e4m3":
            out |= {"sm": opt.exp_avg_scale, "sv": opt.exp_avg_sq_scale}
        if case["clip"]:
            out["norm"] = opt.grad_norm
        return out
    if case["op"] == "norm":
        kind = P.NORM_LAYER if s["layer"] else P.NORM_RMS
        rt = P.DTYPE_FP32 if case["resid"] == "fp32" else P.DTYPE_BF16
        o = s["out"]
        if case["dir"] == "fwd":
            P.osdp_block_norm_fwd(s["x"], s["y"], s["M"], s["D"], rt, kind, s["w_post"], s["b_post"], s["eps"], s["gate"], s["alpha"],
                                  s["beta"], kind, s["w_pre"], s["b_pre"], s["eps"], o[0], o[1], None, o[2], check=True)
            return o
        P.osdp_block_norm_bwd(s["dr"], s["du"], s["y"], s["r"], s["stats"], s["M"], s["D"], rt, kind, s["w_post"], s["b_post"],
                              s["gate"], s["alpha"], s["beta"], kind, s["w_pre"], o["dx"], o["dy"], o["dw_post"], o.get("db_post"),
                              o.get("dgate"), o["dw_pre"], o.get("db_pre"), s["ws"], check=True)
        return o
    return s["layer"](s["x"])


# ---------------------------------------------------------------------------------------------------------------------
# the plain forms

def _statistics(v, layer, eps):
    """[rows, 2]: mean (0 for the RMS norm) and reciprocal deviation."""
    mean = v.mean(1, keepdim=True) if layer else torch.zeros_like(v[:, :1])
    return torch.cat([mean, torch.rsqrt((v - mean).square().mean(1, keepdim=True) + eps)], 1)


def _plain_step(s, lo, hi, wd, coef):
    """One AdamW step on elements [lo, hi) of the flat buffers."""
    h, eight = HYPER, s["m"].dtype == F8
    t = s["steps"]
    g = s["grad"][lo:hi].float()
    if coef is not None:
        g = g * coef
    blocks = slice(lo // QB, hi // QB)
    if eight:
        m = (s["m"][lo:hi].float().view(-1, QB) * s["sm"][blocks, None]).view(-1)
        v = (s["v"][lo:hi].float().view(-1, QB) * s["sv"][blocks, None]).view(-1).square()
    else:
        m, v = s["m"][lo:hi], s["v"][lo:hi]
    m = m * h["b1"] + g * (1.0 - h["b1"])
    v = v * h["b2"] + (g * g) * (1.0 - h["b2"])
    root = v.sqrt()
    p = s["param"] if s["master"] is None else s["master"]
    w = p[lo:hi].float()
    size = h["lr"] / (1.0 - h["b1"] ** t)
    w = w * (1.0 - h["lr"] * wd) - m / (root * (1.0 / math.sqrt(1.0 - h["b2"] ** t)) + h["eps"]) * size
    if s["master"] is not None:
        s["master"][lo:hi] = w
    s["param"][lo:hi] = w.to(s["param"].dtype)
    if eight:
        s["m"][lo:hi], s["sm"][blocks] = _quantise(m, False)
        s["v"][lo:hi], s["sv"][blocks] = _quantise(root, True)
    else:
        s["m"][lo:hi], s["v"][lo:hi] = m, v


def _plain_adamw(s):
    case = s["case"]
    s["steps"] += 1
    coef = None
    out = {"param": s["param"], "m": s["m"], "v": s["v"]}
    if case["clip"]:
        norm = s["grad"].float().square().sum().sqrt()
        coef = torch.clamp(HYPER["max_norm"] / (norm + 1e-6), max=1.0)
        out["norm"] = torch.stack([norm, coef])
    total = s["param"].numel()
    _plain_step(s, 0, s["cut"], HYPER["wd"], coef)
    if s["cut"] < total:
        _plain_step(s, s["cut"], total, 0.0, coef)
    if case["master"]:
        out["master"] = s["master"]
    if case["state"] == "e4m3":
        out |= {"sm": s["sm"], "sv": s["sv"]}
    return out


def _plain_norm_fwd(s):
    y, x = s["y"].float(), s["x"].float()
    sy = _statistics(y, s["layer"], s["eps"])
    p = (y - sy[:, :1]) * sy[:, 1:] * s["w_post"]
    if s["layer"]:
        p = p + s["b_post"]
    if s["gate"] is not None:
        p = p * s["gate"]
    r = s["alpha"] * x + s["beta"] * p
    sr = _statistics(r, s["layer"], s["eps"])
    u = (r - sr[:, :1]) * sr[:, 1:] * s["w_pre"]
    if s["layer"]:
        u = u + s["b_pre"]
    return r.to(s["x"].dtype), u.to(BF16), torch.cat([sy, sr], 1)


def _norm_grad(a, h, rstd, layer):
    d = a - h * (a * h).mean(1, keepdim=True)
    if layer:
        d = d - a.mean(1, keepdim=True)
    return d * rstd


def _plain_norm_bwd(s):
    st, du, layer = s["stats"], s["du"].float(), s["layer"]
    h_pre = (s["r"].float() - st[:, 2:3]) * st[:, 3:4]
    h_post = (s["y"].float() - st[:, 0:1]) * st[:, 1:2]
    t = s["dr"].float() + _norm_grad(du * s["w_pre"], h_pre, st[:, 3:4], layer)
    out = {"dx": (s["alpha"] * t).to(s["dr"].dtype), "dw_pre": (du * h_pre).sum(0)}
    if layer:
        out["db_pre"] = du.sum(0)
    tb = s["beta"] * t
    if s["gate"] is not None:
        p = h_post * s["w_post"]
        if layer:
            p = p + s["b_post"]
        out["dgate"] = (tb * p).sum(0)
        tb = tb * s["gate"]
    out["dw_post"] = (tb * h_post).sum(0)
    if layer:
        out["db_post"] = tb.sum(0)
    out["dy"] = _norm_grad(tb * s["w_post"], h_post, st[:, 1:2], layer).to(BF16)
    return out


def _plain_i8(s):
    x = s["x"].float()
    sx = x.abs().amax(1, keepdim=True) / 127.0
    q = torch.where(sx > 0, torch.round(x / sx), torch.zeros_like(x))
    y = (q @ s["wq"].float().t()) * sx * s["ws"]
    if s["bias"] is not None:
        y = y + s["bias"]
    if s["act"]:
        y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    return y.to(BF16)


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    if op == "adamw":
        return _plain_adamw(state)
    if op == "norm":
        return _plain_norm_fwd(state) if state["case"]["dir"] == "fwd" else _plain_norm_bwd(state)
    return _plain_i8(state)


# ---------------------------------------------------------------------------------------------------------------------

def work(case):
    if case["op"] == "adamw":
        n = sum(_sizes(case)[0])
        e = 2 if case["param"] == "bf16" else 4
        per = 3 * e + (8 if case["master"] else 0) + (16 if case["state"] == "fp32" else 4 + 16.0 / QB)
        return {"bytes": n * per, "flops": n * 16}
    if case["op"] == "norm":
        M, D, e = case["M"], case["D"], 2 if case["resid"] == "bf16" else 4
        n = M * D
        if case["dir"] == "fwd":
            return {"bytes": n * (2 * e + 4) + 16 * M + 20 * D, "flops": n * 14}
        return {"bytes": n * (3 * e + 6) + 16 * M + 32 * D, "flops": n * 28}
    M, N, K = case["M"], case["N"], case["K"]
    return {"bytes": 2 * M * K + N * K + 2 * M * N + 8 * N, "flops": 2 * M * N * K}


def exact(case, seed):
    """The outputs of the first pass in 64 bits, from the definitions."""
    s = _inputs(case, seed)
    D64 = torch.float64
    if case["op"] == "adamw":
        h, t = HYPER, s["steps"] + 1
        total = s["param"].numel()
        wide = lambda c, sc: (c.to(D64).view(-1, QB) * sc.to(D64)[:, None]).view(-1)                # noqa: E731
        g = s["grad"].to(D64)
        out = {}
        if case["clip"]:
            norm = torch.linalg.vector_norm(g)
            coef = min(1.0, h["max_norm"] / (float(norm) + 1e-6))
            out["norm"] = torch.tensor([float(norm), coef], dtype=D64)
            g = g * coef
        eight = case["state"] == "e4m3"
        m = (wide(s["m"], s["sm"]) if eight else s["m"].to(D64)) * h["b1"] + (1 - h["b1"]) * g
        v = (wide(s["v"], s["sv"]).pow_(2) if eight else s["v"].to(D64)) * h["b2"] + (1 - h["b2"]) * g * g
        del g
        w = (s["param"] if s["master"] is None else s["master"]).to(D64)
        w[:s["cut"]] *= 1 - h["lr"] * h["wd"]
        w -= h["lr"] * (m / (1 - h["b1"] ** t)) / (torch.sqrt(v / (1 - h["b2"] ** t)) + h["eps"])
        out["param"] = w
        if case["master"]:
            out["master"] = w
        if not eight:
            return out | {"m": m, "v": v}
        for name, scale, val in (("m", "sm", m), ("v", "sv", v.sqrt_())):
            top = val.view(-1, QB).abs().amax(1)
            top = torch.where(top >= TINY, top, torch.zeros_like(top))
            out[scale] = top / 448
            out[name] = torch.where(top[:, None] > 0, val.view(-1, QB) * 448 / top[:, None], torch.zeros((), dtype=D64, device="cuda")).view(-1)
        assert out["m"].numel() == total
        return out
    if case["op"] == "norm":
        d = {k: (v.to(D64) if torch.is_tensor(v) else v) for k, v in s.items()}
        gate = d["gate"] if d["gate"] is not None else 1.0
        if case["dir"] == "fwd":
            def norm(v, w, b):
                mean = v.mean(1, keepdim=True) if d["layer"] else torch.zeros(v.shape[0], 1, dtype=D64, device="cuda")
                rstd = 1.0 / torch.sqrt((v - mean).pow(2).mean(1, keepdim=True) + d["eps"])
                z = (v - mean) * rstd * w
                return (z + b if d["layer"] else z), torch.cat([mean, rstd], 1)
            p, sy = norm(d["y"], d["w_post"], d["b_post"])
            r = d["alpha"] * d["x"] + d["beta"] * gate * p
            u, sr = norm(r, d["w_pre"], d["b_pre"])
            return r, u, torch.cat([sy, sr], 1)
        # the gradients by their sums over rows and columns; k: elements of a row
        k, (mp, ip, mr, ir) = case["D"], d["stats"].unsqueeze(2).unbind(1)
        hp, hr = (d["y"] - mp) * ip, (d["r"] - mr) * ir
        a = d["du"] * d["w_pre"]
        t = d["dr"] + ir * (a - hr * ((a * hr).sum(1, keepdim=True) / k) - (a.sum(1, keepdim=True) / k if d["layer"] else 0.0))
        out = {"dx": d["alpha"] * t, "dw_pre": torch.einsum("md,md->d", d["du"], hr)}
        c = d["beta"] * torch.einsum("md,md->d", t, hp)
        z = d["beta"] * t.sum(0)
        out["dw_post"] = c * gate
        if d["layer"]:
            out["db_pre"], out["db_post"] = d["du"].sum(0), z * gate
        if d["gate"] is not None:
            out["dgate"] = c * d["w_post"] + (z * d["b_post"] if d["layer"] else 0.0)
        q = t * (d["beta"] * gate * d["w_post"])
        out["dy"] = ip * (q - hp * ((q * hp).sum(1, keepdim=True) / k) - (q.sum(1, keepdim=True) / k if d["layer"] else 0.0))
        return out
    x = s["x"].to(D64)
    top = x.abs().amax(1, keepdim=True)
    q = torch.where(top > 0, torch.round(127.0 * x / top), torch.zeros_like(x))
    y = (q @ s["wq"].to(D64).t()) * (top / 127.0) * s["ws"].to(D64)
    if s["bias"] is not None:
        y = y + s["bias"].to(D64)
    if s["act"]:
        y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)))
    return y
