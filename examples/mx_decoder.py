"""One decoder layer served from microscaled numbers: 4-bit weights and
activations, an 8- or 4-bit paged cache, and attention over it.

    python examples/mx_decoder.py [--fmt fp8] [--steps 16]

Random weights of a grouped-query layer (16 query heads, 4 cache heads of 64,
width 1024, gated MLP of 2816).  Prompts of different lengths are run through it
one after the other: their keys and values are quantized into the cache's pages,
and the prompt attends over what the cache holds (read back).  Then every
sequence decodes token by token: projections of the batch's tokens, one write
into the cache, attention over the pages, output projection and MLP, each by the
library.  The same layer computed in fp32 by torch, from the numbers that
the quantized weights stand for and an unquantized cache, shows what the
quantization of activations and cache costs.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2002_09049_amd import mpq  # noqa: E402

WIDTH, HEADS, KV_HEADS, DIM, INNER = 1024, 16, 4, 64, 2816
PAGE = 32


def norm(x):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


class Layer:
    """Weights as the library holds them, and the fp32 values they stand for."""

    def __init__(self, seed: int):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.held, self.plain = {}, {}
        for name, rows, cols in (("qkv", (HEADS + 2 * KV_HEADS) * DIM, WIDTH), ("out", WIDTH, HEADS * DIM),
                                 ("up", 2 * INNER, WIDTH), ("down", WIDTH, INNER)):
            W = torch.randn((rows, cols), generator=g, device="cuda") / math.sqrt(cols)
            self.held[name] = mpq.mx_quantize(W)
            self.plain[name] = mpq.mx_dequantize(*self.held[name], cols)

    def linear(self, name, x, plain):
        if plain:
            return x @ self.plain[name].t()
        return mpq.mx_linear(x, *self.held[name])

    def qkv(self, x, plain=False):
        h = self.linear("qkv", norm(x), plain).reshape(x.shape[0], HEADS + 2 * KV_HEADS, DIM)
        return h.split([HEADS, KV_HEADS, KV_HEADS], 1)

    def after(self, x, attended, plain=False):
        x = x + self.linear("out", attended.reshape(x.shape[0], -1), plain)
        gate, up = self.linear("up", norm(x), plain).chunk(2, -1)
        return x + self.linear("down", (torch.nn.functional.silu(gate.float()) * up.float()).to(x.dtype), plain)


def attend_prompt(q, k, v):
    """Causal attention of a whole prompt, fp32: q [n, heads, dim]."""
    n = q.shape[0]
    k, v = (t.float().repeat_interleave(HEADS // KV_HEADS, 1).transpose(0, 1).contiguous() for t in (k, v))
    s = q.float().transpose(0, 1).contiguous() @ k.transpose(1, 2).contiguous() / math.sqrt(DIM)
    s = s.masked_fill(torch.ones((n, n), dtype=torch.bool, device=s.device).triu(1), -math.inf)
    return (torch.softmax(s, -1) @ v).transpose(0, 1).to(q.dtype)


def run(fmt: str = "fp8", prompts=(7, 150, 64, 33), steps: int = 16, seed: int = 0):
    """Decodes `steps` tokens of every sequence.  Returns (outputs [steps,
    batch, width], the fp32 layer's outputs of the same inputs)."""
    layer = Layer(seed)
    batch = len(prompts)
    most = -(-(max(prompts) + steps) // PAGE)
    cache = mpq.MXCache.empty(batch * most + 1, PAGE, KV_HEADS, DIM, fmt)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    table = torch.randperm(batch * most, generator=g, device="cuda").to(torch.int32).reshape(batch, most)
    wide = table.long()

    def slots_of(b, tokens):
        return wide[b, tokens // PAGE] * PAGE + tokens % PAGE

    past = []                       # the fp32 layer's keys and values, sequence by sequence
    for b, n in enumerate(prompts):
        x = torch.randn((n, WIDTH), generator=g, device="cuda").bfloat16()
        q, k, v = layer.qkv(x)
        slots = slots_of(b, torch.arange(n, device="cuda"))
        cache.write(k, v, slots)
        layer.after(x, attend_prompt(q, *cache.read(slots, dtype=torch.bfloat16)))
        past.append([list(t) for t in layer.qkv(x.float(), plain=True)[1:]])

    space = torch.empty((max(1, cache.attend_workspace(batch, HEADS, most)),), dtype=torch.uint8, device="cuda")
    lengths = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    rows = torch.arange(batch, device="cuda")
    outs, plains = [], []
    for _ in range(steps):
        x = torch.randn((batch, WIDTH), generator=g, device="cuda").bfloat16()
        q, k, v = layer.qkv(x)
        cache.write(k, v, slots_of(rows, lengths.long()))
        lengths = lengths + 1
        outs.append(layer.after(x, cache.attend(q, table, lengths, workspace=space)))

        qp, kp, vp = layer.qkv(x.float(), plain=True)
        attended = []
        for b in range(batch):
            past[b][0].append(kp[b])
            past[b][1].append(vp[b])
            ks, vs = (torch.stack(t).repeat_interleave(HEADS // KV_HEADS, 1) for t in past[b])
            p = torch.softmax((ks * qp[b]).sum(-1) / math.sqrt(DIM), 0)
            attended.append((p[..., None] * vs).sum(0))
        plains.append(layer.after(x.float(), torch.stack(attended), plain=True))
    return torch.stack(outs).float(), torch.stack(plains)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--fmt", choices=sorted(mpq.MX_FORMATS), default="fp8")
    ap.add_argument("--steps", type=int, default=16)
    a = ap.parse_args()
    got, want = run(a.fmt, steps=a.steps)
    torch.cuda.synchronize()
    err = ((got - want).norm(dim=-1) / want.norm(dim=-1))
    print(f"{a.steps} steps of {got.shape[1]} sequences, cache {a.fmt}: relative error to the fp32 layer "
          f"mean {err.mean():.4f}, largest {err.max():.4f}")


if __name__ == "__main__":
    main()
