#!/usr/bin/env python3
"""Trains a stack of residual MLP blocks and serves it in int8.

    python examples/residual_blocks.py [--hidden 512] [--ffn 2048] [--blocks 4] [--tokens 2048] [--steps 200] [--experts 0]

A block is  r = x + gate (.) N(MLP(u)),  u' = N'(r): the split MLP (its weights in one flat parameter buffer) between
fused norms, gate and residual sum (``nn.ResidualNorm``).  All parameters, flat bf16 buffers and fp32 vectors, are
stepped by ``optim.AdamW``: the bf16 ones with fp32 masters and 8-bit states, all gradients clipped by one norm on the
device.  The trained blocks are then run with int8 weights (``nn.Int8Linear``), the norms handing their output over as
int8 with a scale per token, for a batch and for a single token.  The task is to reproduce a fixed random network of the same form.

With --experts E the blocks of the student are mixtures of E MLPs, of which every token takes two (``nn.ExpertMLP`` behind a gate and
``nn.ExpertRouter``); they are trained alike and not served in int8.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2209_13258_b200 as P                                          # noqa: E402
from paper_2209_13258_b200.nn import ExpertMLP, ExpertRouter, Int8Linear, ResidualNorm, SplitLinear, SplitMLP    # noqa: E402
from paper_2209_13258_b200.optim import AdamW, ClippedStep                 # noqa: E402


class ExpertBlock(torch.nn.Module):
    """A mixture of MLPs with its gate."""

    def __init__(self, hidden, ffn, experts, top_k=2):
        super().__init__()
        self.gate = SplitLinear(hidden, -(-experts // 8) * 8, bias=False)     # (its outputs come in eights; those over are left out)
        self.router, self.mlp = ExpertRouter(experts, top_k), ExpertMLP(hidden, ffn, experts)

    def forward(self, u):
        return self.mlp(u, *self.router(self.gate(u)[..., :self.router.experts]))


class Stack(torch.nn.Module):
    def __init__(self, hidden, ffn, blocks, k_split=2, experts=0):
        super().__init__()
        self.first = ResidualNorm(hidden, post=None, pre="rms", gate=False, resid_dtype=torch.float32)
        self.mlps = torch.nn.ModuleList(ExpertBlock(hidden, ffn, experts) if experts else SplitMLP(hidden, ffn, k_split=k_split) for _ in range(blocks))
        # behind the last block there is no norm for a next one
        self.norms = torch.nn.ModuleList(
            ResidualNorm(hidden, post="rms", pre="rms" if b + 1 < blocks else None, gate_init=0.5, resid_dtype=torch.float32)
            for b in range(blocks))

    def forward(self, x):
        x, u = self.first(x)
        for mlp, norm in zip(self.mlps, self.norms):
            x, u = norm(x, mlp(u))
        return x


class Int8Stack:
    """The same blocks with int8 weights and activations."""

    def __init__(self, stack):
        self.first, self.norms = stack.first, stack.norms
        mk = lambda w, b, act: Int8Linear(*_quantised(w), b.detach().clone(), act=act)      # noqa: E731
        self.layers = [(mk(m.w1, m.b1, m.act), mk(m.w2, m.b2, P.ACT_NONE)) for m in stack.mlps]

    def __call__(self, x):
        x, u = self.first.forward_int8(x)
        for (up, down), norm in zip(self.layers, self.norms):
            y = down(up(u))
            if norm.pre == P.NORM_NONE:
                with torch.no_grad():
                    return norm(x, y)[0]
            x, u = norm.forward_int8(x, y)


def _quantised(w):
    from paper_2209_13258_b200.nn import quantize_int8
    return quantize_int8(w)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--hidden", type=int, default=512)
    ap.add_argument("--ffn", type=int, default=2048)
    ap.add_argument("--blocks", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--lr", type=float, default=2e-3)
    ap.add_argument("--experts", type=int, default=0)
    a = ap.parse_args(argv)
    torch.manual_seed(0)
    teacher, student = Stack(a.hidden, a.ffn, a.blocks), Stack(a.hidden, a.ffn, a.blocks, experts=a.experts)
    for p in teacher.parameters():
        p.requires_grad_(False)
    half = [p for p in student.parameters() if p.dtype == torch.bfloat16]
    full = [p for p in student.parameters() if p.dtype == torch.float32]
    # bf16 and fp32 parameters have their own optimisers, and one gradient norm
    opt = ClippedStep([AdamW(half, lr=a.lr, weight_decay=0.01, state_dtype="e4m3", master=True), AdamW(full, lr=a.lr, weight_decay=0.0)],
                      max_norm=1.0)
    losses = []
    for step in range(a.steps):
        x = torch.randn(a.tokens, a.hidden, device="cuda")
        with torch.no_grad():
            want = teacher(x)
        loss = (student(x) - want).square().mean()
        loss.backward()
        opt.step()
        opt.zero_grad()
        if step % max(1, a.steps // 10) == 0 or step == a.steps - 1:
            losses.append(float(loss.detach()))
            print("step %4d  loss %.5f  gradient norm %.4f" % (step, losses[-1], float(opt.grad_norm[0])))
    if a.experts:
        return losses, {}
    served = Int8Stack(student)
    errors = {}
    for tokens in (64, 1):
        x = torch.randn(tokens, a.hidden, device="cuda")
        with torch.no_grad():
            ref = student(x)
        moved = (ref - x).norm()                  # what the blocks add to the stream
        errors[tokens] = float((served(x) - ref).norm() / moved)
        print("int8, %d token(s): error %.4f of what the blocks add" % (tokens, errors[tokens]))
    return losses, errors


if __name__ == "__main__":
    main()
