"""Workloads of the mixture-of-experts operators: routing (forward and backward), the plan with dispatch and combine of the
experts' rows, and the experts' products (forward, backward, and for a few tokens).

`run` computes them in elementary torch operations, or, with `own` set, with this package's kernels.

Layout of the experts' rows: expert e has `count[e]` rows from row `offset[e]`, a multiple of 64, in the order of its
(token, choice) pairs; the rows up to the next expert's are zero, rows behind the last expert's are left as they were.
"""
import math
import random

import torch

own = False

F32, F64, BF16 = torch.float32, torch.float64, torch.bfloat16
ROWS = 64           # an expert's rows start at a multiple of this


def listed():
    return [
        # --- routing ---
        # one token while a sequence is generated: a call whose cost is its launch
        {"name": "route-token", "op": "route", "dir": "fwd", "T": 1, "E": 64, "k": 2, "score": "softmax", "renorm": True, "logits": "bf16",
         "bias": False, "groups": 1, "top_groups": 1, "take": 1},
        # a training batch with many experts, a bias for balance, and the choice limited to four groups of eight
        {"name": "route-16384-groups", "op": "route", "dir": "fwd", "T": 16384, "E": 256, "k": 8, "score": "sigmoid", "renorm": True,
         "logits": "fp32", "bias": True, "groups": 8, "top_groups": 4, "take": 2},
        # ragged batch, a number of experts that is no power of two, every logit has a gradient
        {"name": "route-bwd-ragged", "op": "route", "dir": "bwd", "T": 1777, "E": 60, "k": 4, "score": "softmax", "renorm": False, "logits": "bf16"},
        # backward of the large training batch
        {"name": "route-bwd-16384", "op": "route", "dir": "bwd", "T": 16384, "E": 256, "k": 8, "score": "sigmoid", "renorm": True, "logits": "fp32"},
        # --- the experts' rows ---
        # plan and dispatch of a training batch of the hidden-2048 model
        {"name": "dispatch-2048", "op": "rows", "dir": "dispatch", "T": 8192, "E": 8, "k": 2, "D": 2048},
        # ragged batch of a narrow model: what the weighted sum sends back, with the gradient of its weights
        {"name": "combine-bwd-ragged", "op": "rows", "dir": "combine-bwd", "T": 1777, "E": 60, "k": 4, "D": 1032},
        # the weighted sum of the wide model's training batch
        {"name": "combine-8192", "op": "rows", "dir": "combine", "T": 16384, "E": 8, "k": 2, "D": 8192},
        # --- the experts' products ---
        # one token through the first layer of its two experts: reading their weights once is the whole cost
        {"name": "linear-token", "op": "linear", "dir": "fwd", "T": 1, "E": 8, "k": 2, "N": 8192, "K": 2048, "act": True, "bias": True},
        # a handful of sequences, odd batch, more experts than most of them need
        {"name": "linear-batch-37", "op": "linear", "dir": "fwd", "T": 37, "E": 16, "k": 2, "N": 2064, "K": 1032, "act": False, "bias": True},
        # a training batch of the hidden-2048 model through the first layer
        {"name": "linear-2048", "op": "linear", "dir": "fwd", "T": 8192, "E": 8, "k": 2, "N": 8192, "K": 2048, "act": True, "bias": True},
        # many narrow experts, none with a round number of rows: backward of the first layer
        {"name": "linear-bwd-ragged", "op": "linear", "dir": "bwd", "T": 1777, "E": 60, "k": 4, "N": 2064, "K": 1032, "act": True, "bias": True},
        # the wide model's second layer, backward
        {"name": "linear-bwd-wide", "op": "linear", "dir": "bwd", "T": 8192, "E": 4, "k": 2, "N": 8192, "K": 32768, "act": False, "bias": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _extent(rng, lo, hi):
    """A multiple of 8 in [lo, hi], spread over the logarithm."""
    return max(lo // 8, min(hi // 8, round(_log(rng, lo, hi) / 8))) * 8


def draw(rng):
    op = rng.choice(["route", "rows", "linear"])
    T, k = _log(rng, 1, 16384), rng.choice([1, 2, 2, 3, 4, 6, 8])
    if op == "route":
        groups = rng.choice([1, 1, 4, 8])
        E = max(k, _log(rng, 2, 256))
        E = -(-E // groups) * groups
        E = max(E, 2 * groups) if groups > 1 else E
        top = max(-(-k // (E // groups)), rng.randint(1, groups))
        c = {"op": op, "dir": rng.choice(["fwd", "bwd"]), "T": T, "E": E, "k": k, "score": rng.choice(["softmax", "sigmoid"]),
             "renorm": rng.random() < 0.6, "logits": rng.choice(["bf16", "fp32"])}
        return c if c["dir"] == "bwd" else c | {"bias": rng.random() < 0.5, "groups": groups, "top_groups": top, "take": rng.choice([1, 2])}
    E = max(k, _log(rng, 2, 256))
    if op == "rows":
        D = _extent(rng, 64, 8192)
        T = max(1, min(T, 16384 * 8192 * 2 // (D * k)))
        return {"op": op, "dir": rng.choice(["dispatch", "combine", "combine-bwd"]), "T": T, "E": E, "k": k, "D": D}
    N, K = _extent(rng, 64, 8192), _extent(rng, 64, 8192)
    while E > k and E * N * K > 1 << 29:
        E = max(k, E // 2)
    T = max(1, min(T, (1 << 38) // (k * N * K)))
    return {"op": op, "dir": rng.choice(["fwd", "bwd"]), "T": T, "E": E, "k": k, "N": N, "K": K, "act": rng.random() < 0.5, "bias": rng.random() < 0.7}


# ---------------------------------------------------------------------------------------------------------------------
# inputs

def _dtype(name):
    return {"bf16": BF16, "fp32": F32}[name]


SCALE = 2.5         # what the weights of a token are scaled to


def _row_count(T, k, E):
    """Rows that are enough however the choices fall."""
    return (T * k + (ROWS - 1) * min(E, T * k)) // ROWS * ROWS


def _layout(idx, E):
    """Counts and first rows of the experts [E], row of every (token, choice) [T, k]."""
    flat = idx.reshape(-1).long()
    counts = torch.zeros(E, dtype=torch.int64, device=idx.device).scatter_add_(0, flat, torch.ones_like(flat))
    padded = (counts + ROWS - 1) // ROWS * ROWS
    offsets = padded.cumsum(0) - padded
    order = torch.argsort(flat, stable=True)
    expert = flat[order]
    rank = torch.arange(flat.numel(), device=idx.device) - (counts.cumsum(0) - counts)[expert]
    pos = torch.empty_like(flat)
    pos[order] = offsets[expert] + rank
    return counts, offsets, pos.view(idx.shape)


def _choices(g, T, E, k):
    """Experts of T tokens, some experts more popular than others."""
    popular = 0.4 * torch.randn(E, device="cuda", generator=g)
    noise = torch.rand(T, E, device="cuda", generator=g).clamp_(1e-6, 1.0 - 1e-6)
    return torch.sort(popular - torch.log(-torch.log(noise)), dim=1, descending=True, stable=True)[1][:, :k].to(torch.int32).contiguous()


def _inputs(case, seed):
    """What both forms start from."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    rnd = lambda *n: torch.randn(*n, device="cuda", generator=g)                                    # noqa: E731
    T, E, k = case["T"], case["E"], case["k"]
    s = {"case": case}
    if case["op"] == "route":
        s["logits"] = (1.2 * rnd(T, E) + 0.3 * rnd(E)).to(_dtype(case["logits"]))
        if case["dir"] == "fwd":
            s["bias"] = 0.05 * rnd(E) if case["bias"] else None
            return s
        scores = s["logits"].to(F64)
        s["idx"] = torch.sort(scores, dim=1, descending=True, stable=True)[1][:, :k].to(torch.int32).contiguous()
        s["dweights"] = rnd(T, k)
        return s
    s["idx"] = _choices(g, T, E, k)
    R = s["R"] = _row_count(T, k, E)
    counts, offsets, pos = _layout(s["idx"], E)
    if case["op"] == "rows":
        D = case["D"]
        if case["dir"] == "dispatch":
            s["x"] = rnd(T, D).to(BF16)
            return s
        s["pos"], s["weights"] = pos, torch.rand(T, k, device="cuda", generator=g) * (2.0 / k) + 0.05
        s["y"] = torch.zeros(R, D, dtype=BF16, device="cuda")
        s["y"][pos.view(-1)] = rnd(T * k, D).to(BF16)
        if case["dir"] == "combine-bwd":
            s["dout"] = rnd(T, D).to(BF16)
            s["counts"], s["offsets"] = counts, offsets
        return s
    N, K = case["N"], case["K"]
    s["x"] = torch.zeros(R, K, dtype=BF16, device="cuda")
    tokens = rnd(T, K).to(BF16)
    s["x"][pos.view(-1)] = tokens.repeat_interleave(k, 0)
    s["w"] = torch.empty(E, N, K, dtype=BF16, device="cuda")
    for e in range(E):
        s["w"][e] = rnd(N, K).mul_(K ** -0.5)
    s["bias"] = 0.1 * rnd(E, N) if case["bias"] else None
    if case["dir"] == "bwd":
        s["dy"] = torch.zeros(R, N, dtype=BF16, device="cuda")
        s["dy"][pos.view(-1)] = (0.1 * rnd(T * k, N)).to(BF16)
        s["z"] = None
        if case["act"]:
            s["z"] = torch.zeros(R, N, dtype=BF16, device="cuda")
            s["z"][pos.view(-1)] = rnd(T * k, N).to(BF16)
    # experts that have rows, and their rows as a table [live, most] (R where there is none): what the plan tells the plain form
    most = int(counts.max())
    s["live"] = counts.nonzero().view(-1)
    at = torch.arange(most, device="cuda")
    s["table"] = torch.where(at < counts[s["live"], None], offsets[s["live"], None] + at, R)
    s["counts"], s["offsets"] = counts, offsets
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    # what a program keeps between calls: output buffers, the plan of the batch, the workspace
    import paper_2209_13258_b200 as P
    T, E, k = case["T"], case["E"], case["k"]
    new = lambda dt, *n: torch.zeros(*n, dtype=dt, device="cuda")                                   # noqa: E731
    if case["op"] == "route":
        if case["dir"] == "fwd":
            s["out"] = new(torch.int32, T, k), new(F32, T, k)
        else:
            s["out"] = torch.empty_like(s["logits"])
        return s
    R, plan_ints = P.osdp_expert_rows(T, k, E)[1:]
    assert R == s["R"]
    s["plan"], s["pos"] = new(torch.int32, plan_ints), new(torch.int32, T, k)
    P.osdp_expert_plan(s["idx"], T, k, E, s["plan"], s["pos"], check=True)
    if case["op"] == "rows":
        D = case["D"]
        s["rows"] = new(BF16, R, D)
        s["out"] = new(BF16, T, D)
        s["dweights"] = new(F32, T, k)
        return s
    N, K = case["N"], case["K"]
    act = s["act"] = P.ACT_GELU_TANH if case["act"] else P.ACT_NONE
    op = P.OP_LINEAR_FWD if case["dir"] == "fwd" else P.OP_LINEAR_BWD
    s["ws"] = P.new_workspace(P.osdp_expert_linear_workspace_bytes(T, k, E, N, K, act, op)[1])
    if case["dir"] == "fwd":
        s["out"] = new(BF16, R, N)
    else:
        s["out"] = {"dx": new(BF16, R, K), "dw": new(BF16, E, N, K)}
        if case["bias"]:
            s["out"]["db"] = new(F32, E, N)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# the framework's calls

def _run_own(s):
    import paper_2209_13258_b200 as P
    case = s["case"]
    T, E, k = case["T"], case["E"], case["k"]
    if case["op"] == "route":
        score = P.SCORE_SOFTMAX if case["score"] == "softmax" else P.SCORE_SIGMOID
        dt = P.DTYPE_FP32 if case["logits"] == "fp32" else P.DTYPE_BF16
        if case["dir"] == "fwd":
            idx, weights = s["out"]
            P.osdp_route_fwd(s["logits"], E, dt, s["bias"], T, E, k, score, case["groups"], case["top_groups"], case["take"],
                             case["renorm"], SCALE, idx, weights, check=True)
        else:
            P.osdp_route_bwd(s["dweights"], s["logits"], E, dt, s["idx"], T, E, k, score, case["renorm"], SCALE, s["out"], E, check=True)
        return s["out"]
    plan, pos = s["plan"], s["pos"]
    if case["op"] == "rows":
        D = case["D"]
        if case["dir"] == "dispatch":
            P.osdp_expert_plan(s["idx"], T, k, E, plan, pos, check=True)
            P.osdp_expert_dispatch(s["x"], plan, pos, None, None, T, k, E, D, s["rows"], None, check=True)
            return {"pos": pos, "rows": s["rows"]}
        if case["dir"] == "combine":
            P.osdp_expert_combine(s["y"], plan, pos, s["weights"], T, k, E, D, s["out"], check=True)
            return s["out"]
        P.osdp_expert_dispatch(s["dout"], plan, pos, s["weights"], s["y"], T, k, E, D, s["rows"], s["dweights"], check=True)
        return {"dy": s["rows"], "dweights": s["dweights"]}
    N, K = case["N"], case["K"]
    if case["dir"] == "fwd":
        P.osdp_expert_linear_fwd(s["x"], plan, s["w"], 0, s["bias"], T, k, E, N, K, s["act"], s["out"], None, s["ws"], check=True)
        return s["out"]
    o = s["out"]
    P.osdp_expert_linear_bwd(s["dy"], s["x"], plan, s["w"], 0, s["z"], T, k, E, N, K, s["act"], o["dx"], o["dw"], 0, P.DTYPE_BF16, 0,
                             o.get("db"), s["ws"], check=True)
    return o


# ---------------------------------------------------------------------------------------------------------------------
# the plain forms

def _scores(logits, case):
    return torch.softmax(logits, 1) if case["score"] == "softmax" else torch.sigmoid(logits)


def _plain_route(s):
    case = s["case"]
    T, E, k = case["T"], case["E"], case["k"]
    score = _scores(s["logits"].to(F64), case)        # in 64 bits: values next to one another decide which expert is taken
    choice = score if s["bias"] is None else score + s["bias"].to(F64)
    if case["top_groups"] < case["groups"]:
        per = choice.view(T, case["groups"], -1)
        best = torch.sort(per, dim=2, descending=True)[0][:, :, :case["take"]].sum(2)
        rank = torch.argsort(torch.argsort(best, dim=1, descending=True, stable=True), dim=1)
        choice = torch.where((rank < case["top_groups"])[:, :, None], per, -math.inf).view(T, E)
    idx = torch.sort(choice, dim=1, descending=True, stable=True)[1][:, :k]
    w = score.gather(1, idx)
    if case["renorm"]:
        w = w / w.sum(1, keepdim=True)
    return idx.to(torch.int32), (w * SCALE).to(F32)


def _plain_route_bwd(s):
    case = s["case"]
    score = _scores(s["logits"].float(), case)
    idx = s["idx"].long()
    mine, ds = score.gather(1, idx), s["dweights"] * SCALE
    if case["renorm"]:
        total = mine.sum(1, keepdim=True)
        ds = (ds - (ds * mine).sum(1, keepdim=True) / total) / total
    dscore = torch.zeros_like(score).scatter_(1, idx, ds)
    if case["score"] == "softmax":
        d = score * (dscore - (ds * mine).sum(1, keepdim=True))
    else:
        d = dscore * score * (1.0 - score)
    return d.to(s["logits"].dtype)


def _plain_rows(s):
    case = s["case"]
    T, E, k, D = case["T"], case["E"], case["k"], case["D"]
    rows = torch.zeros(s["R"], D, dtype=BF16, device="cuda")
    if case["dir"] == "dispatch":
        pos = _layout(s["idx"], E)[2]
        rows[pos.view(-1)] = s["x"][:, None, :].expand(T, k, D).reshape(T * k, D)
        return {"pos": pos.to(torch.int32), "rows": rows}
    mine = s["y"][s["pos"].view(-1)].view(T, k, D).float()
    if case["dir"] == "combine":
        return (mine * s["weights"][:, :, None]).sum(1).to(BF16)
    dout = s["dout"].float()[:, None, :]
    rows[s["pos"].view(-1)] = (dout * s["weights"][:, :, None]).to(BF16).view(T * k, D)
    return {"dy": rows, "dweights": (dout * mine).sum(2)}


GELU_A, GELU_B = math.sqrt(2.0 / math.pi), 0.044715


def _gelu(z):
    return 0.5 * z * (1.0 + torch.tanh(GELU_A * (z + GELU_B * z * z * z)))


def _gelu_grad(z):
    t = torch.tanh(GELU_A * (z + GELU_B * z * z * z))
    return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * GELU_A * (1.0 + 3.0 * GELU_B * z * z)


def _plain_linear(s):
    case, table, live = s["case"], s["table"], s["live"]
    R = s["R"]
    there = (table < R)[:, :, None]
    at = table.clamp(max=R - 1)
    take = lambda v: torch.where(there, v[at].float(), 0.0)                                         # noqa: E731

    def give(v):
        out = torch.zeros(R + 1, v.shape[2], dtype=BF16, device="cuda")
        out[table] = torch.where(there, v, 0.0).to(BF16)
        return out[:R]
    x, w = take(s["x"]), s["w"][live].float()
    if case["dir"] == "fwd":
        y = torch.bmm(x, w.transpose(1, 2))
        if s["bias"] is not None:
            y = y + s["bias"][live][:, None, :]
        return give(_gelu(y) if case["act"] else y)
    g = take(s["dy"])
    if case["act"]:
        g = g * _gelu_grad(take(s["z"]))
    out = {"dx": give(torch.bmm(g, w)), "dw": torch.zeros_like(s["w"])}
    out["dw"][live] = torch.bmm(g.transpose(1, 2), x).to(BF16)
    if case["bias"]:
        out["db"] = torch.zeros(case["E"], case["N"], device="cuda")
        out["db"][live] = g.sum(1)
    return out


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    if case["op"] == "route":
        return _plain_route(state) if case["dir"] == "fwd" else _plain_route_bwd(state)
    return _plain_rows(state) if case["op"] == "rows" else _plain_linear(state)


# ---------------------------------------------------------------------------------------------------------------------

def work(case):
    T, E, k = case["T"], case["E"], case["k"]
    if case["op"] == "route":
        e = 4 if case["logits"] == "fp32" else 2
        if case["dir"] == "fwd":
            return {"bytes": T * (E * e + 8 * k), "flops": T * E * 8}
        # without the other scores in the gradient only the chosen logits are needed
        reads = E * e if case["score"] == "softmax" and not case["renorm"] else k * e
        return {"bytes": T * (E * e + reads + 8 * k), "flops": T * E * 4}
    n = T * k
    if case["op"] == "rows":
        D = case["D"]
        if case["dir"] == "dispatch":
            return {"bytes": 2 * D * (T + n) + 8 * n, "flops": 4 * n}
        if case["dir"] == "combine":
            return {"bytes": 2 * D * (T + n) + 8 * n, "flops": 2 * n * D}
        return {"bytes": 2 * D * (T + 2 * n) + 12 * n, "flops": 3 * n * D}
    N, K = case["N"], case["K"]
    used = E * (1.0 - (1.0 - k / E) ** T)             # experts that have a row, were they equally popular
    weights = int(used * N * K) * 2
    if case["dir"] == "fwd":
        return {"bytes": weights + 2 * n * (N + K) + int(used) * 4 * N, "flops": 2 * n * N * K}
    return {"bytes": weights + 2 * E * N * K + 2 * n * ((2 if case["act"] else 1) * N + 2 * K) + (4 * E * N if case["bias"] else 0),
            "flops": 4 * n * N * K}


def exact(case, seed):
    """The outputs in 64 bits, from the definitions."""
    s = _inputs(case, seed)
    T, E, k = case["T"], case["E"], case["k"]
    if case["op"] == "route":
        l = s["logits"].to(F64)
        if case["score"] == "softmax":
            p = torch.exp(l - l.max(1, keepdim=True)[0])
            p = p / p.sum(1, keepdim=True)
        else:
            p = 1.0 / (1.0 + torch.exp(-l))
        if case["dir"] == "fwd":
            c = p + (s["bias"].to(F64) if s["bias"] is not None else 0.0)
            if case["top_groups"] < case["groups"]:
                size = E // case["groups"]
                tops = torch.stack([torch.sort(c[:, a:a + size], dim=1, descending=True)[0][:, :case["take"]].sum(1)
                                    for a in range(0, E, size)], 1)
                out = torch.ones_like(tops, dtype=torch.bool)
                for _ in range(case["top_groups"]):
                    best = torch.where(out, tops, -math.inf).max(1, keepdim=True)[0]
                    first = ((tops == best) & out).to(torch.int8).argmax(1, keepdim=True)
                    out.scatter_(1, first, False)
                c = torch.where(out.repeat_interleave(size, 1), -math.inf, c)
            idx = []
            for _ in range(k):
                best = (c == c.max(1, keepdim=True)[0]).to(torch.int8).argmax(1, keepdim=True)
                idx.append(best)
                c = c.scatter(1, best, -math.inf)
            idx = torch.cat(idx, 1)
            w = torch.gather(p, 1, idx)
            return idx.to(torch.int32), SCALE * w / (w.sum(1, keepdim=True) if case["renorm"] else 1.0)
        # derivatives of the weights by the scores, and of the scores by the logits, as matrices applied one after the other
        idx, dw = s["idx"].long(), s["dweights"].to(F64)
        q = torch.gather(p, 1, idx)
        if case["renorm"]:
            total = q.sum(1)[:, None]
            jac = torch.eye(k, dtype=F64, device="cuda")[None] / total[:, :, None] - q[:, :, None] / (total * total)[:, :, None]
            dq = SCALE * torch.einsum("tj,tji->ti", dw, jac)
        else:
            dq = SCALE * dw
        dp = torch.zeros_like(p)
        dp.scatter_add_(1, idx, dq)
        if case["score"] == "softmax":
            return p * dp - p * torch.einsum("te,te->t", p, dp)[:, None]
        return dp * p * (1.0 - p)
    counts, offsets, pos = _layout(s["idx"], E)
    R = s["R"]
    if case["op"] == "rows":
        D = case["D"]
        rows = torch.zeros(R, D, dtype=F64, device="cuda")
        if case["dir"] == "dispatch":
            for j in range(k):
                rows[pos[:, j]] = s["x"].to(F64)
            return {"pos": pos.to(torch.int32), "rows": rows}
        w = s["weights"].to(F64)
        if case["dir"] == "combine":
            out = torch.zeros(T, D, dtype=F64, device="cuda")
            for j in range(k):
                out.add_(s["y"][pos[:, j]].to(F64).mul_(w[:, j, None]))
            return out
        dout, dw = s["dout"].to(F64), torch.empty(T, k, dtype=F64, device="cuda")
        for j in range(k):
            rows[pos[:, j]] = dout * w[:, j, None]
            dw[:, j] = torch.einsum("td,td->t", dout, s["y"][pos[:, j]].to(F64))
        return {"dy": rows, "dweights": dw}
    N, K = case["N"], case["K"]
    first, many = offsets.tolist(), counts.tolist()
    if case["dir"] == "fwd":
        y = torch.zeros(R, N, dtype=F64, device="cuda")
    else:
        out = {"dx": torch.zeros(R, K, dtype=F64, device="cuda"), "dw": torch.zeros(E, N, K, dtype=F64, device="cuda")}
        if case["bias"]:
            out["db"] = torch.zeros(E, N, dtype=F64, device="cuda")
    for e in range(E):
        mine = slice(first[e], first[e] + many[e])
        if many[e] == 0:
            continue
        x, w = s["x"][mine].to(F64), s["w"][e].to(F64)
        if case["dir"] == "fwd":
            z = x @ w.t()
            if s["bias"] is not None:
                z += s["bias"][e].to(F64)
            y[mine] = z / (1.0 + torch.exp(-2.0 * GELU_A * (z + GELU_B * z ** 3))) if case["act"] else z
            continue
        g = s["dy"][mine].to(F64)
        if case["act"]:
            z = s["z"][mine].to(F64)
            u = GELU_A * (z + GELU_B * z ** 3)
            h = 1.0 / (1.0 + torch.exp(-2.0 * u))
            g = g * (h + z * 2.0 * h * (1.0 - h) * GELU_A * (1.0 + 3.0 * GELU_B * z ** 2))
        out["dx"][mine] = g @ w
        out["dw"][e] = g.t() @ x
        if case["bias"]:
            out["db"][e] = g.sum(0)
    return y if case["dir"] == "fwd" else out
