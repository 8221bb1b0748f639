"""One decoder layer with experts served from microscaled numbers: 4-bit weights
and activations, a paged 8- or 4-bit cache, rotated keys and a layer of experts.

    python examples/mx_expert_decoder.py [--fmt fp8] [--steps 16]

Random weights of a grouped-query layer (16 query heads, 4 cache heads of 64,
width 1024) with 12 experts of width 352, three for each token.  All prompts'
tokens lie behind each other and go through in one step: their pages and slots
are planned on the GPU, queries and keys are normed and rotated, keys and
values quantized into the cache, and each prompt attends over what the cache holds
(read back).  Then every sequence decodes token by token, all by the library but for
attention's input norm and the experts' activation.  The same layer computed in fp32
by torch, from the numbers that the quantized weights stand for, an unquantized
cache and the same choices of experts, shows what quantization costs.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2002_09049_amd import mpq  # noqa: E402

WIDTH, HEADS, KV_HEADS, DIM = 1024, 16, 4, 64
EXPERTS, CHOICES, INNER = 12, 3, 352
PAGE, THETA, EPS = 32, 10000.0, 1e-6


def norm(x):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + EPS)).to(x.dtype)


class Layer:
    """Weights as the library holds them, and the fp32 values they stand for."""

    def __init__(self, seed: int):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.held, self.plain = {}, {}
        for name, experts, rows, cols in (("qkv", 1, (HEADS + 2 * KV_HEADS) * DIM, WIDTH), ("out", 1, WIDTH, HEADS * DIM),
                                          ("up", EXPERTS, 2 * INNER, WIDTH), ("down", EXPERTS, WIDTH, INNER)):
            W = torch.randn((experts * rows, cols), generator=g, device="cuda") / math.sqrt(cols)
            codes, scales = mpq.mx_quantize(W)
            plain = mpq.mx_dequantize(codes, scales, cols)
            if experts > 1:
                codes, scales, plain = (t.reshape(experts, rows, -1) for t in (codes, scales, plain))
            self.held[name], self.plain[name] = (codes, scales), plain
        self.router = torch.randn((EXPERTS, WIDTH), generator=g, device="cuda") / math.sqrt(WIDTH)
        self.q_weight, self.k_weight = (torch.rand((DIM,), generator=g, device="cuda") + 0.5 for _ in "qk")
        self.freqs = THETA ** (-torch.arange(0, DIM, 2, dtype=torch.float64, device="cuda") / DIM)

    def qkv(self, x):
        h = mpq.mx_linear(norm(x), *self.held["qkv"]).reshape(x.shape[0], HEADS + 2 * KV_HEADS, DIM)
        return h.split([HEADS, KV_HEADS, KV_HEADS], 1)

    def after(self, x, attended):
        """The rest of the layer; (its output, the experts that were chosen)."""
        x = x + mpq.mx_linear(attended.reshape(x.shape[0], -1), *self.held["out"])
        h = norm(x)
        chosen, weights, order, place, offsets = mpq.mx_route(h.float() @ self.router.t(), CHOICES)
        gate, up = mpq.mx_experts(h, *self.held["up"], offsets, order, CHOICES).chunk(2, -1)
        y = mpq.mx_experts((torch.nn.functional.silu(gate.float()) * up.float()).to(x.dtype), *self.held["down"], offsets)
        return mpq.mx_combine(y, place, weights, x), chosen

    # ---- the same in fp32

    def turned(self, x, positions, weight):
        angle = (positions.double()[:, None] * self.freqs)[:, None]
        a, b = (norm(x) * weight).double().chunk(2, -1)
        return torch.cat((a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()), -1).float()

    def plain_qkv(self, x, positions):
        h = (norm(x) @ self.plain["qkv"][:, :WIDTH].t()).reshape(x.shape[0], HEADS + 2 * KV_HEADS, DIM)
        q, k, v = h.split([HEADS, KV_HEADS, KV_HEADS], 1)
        return self.turned(q, positions, self.q_weight), self.turned(k, positions, self.k_weight), v

    def plain_after(self, x, attended, chosen):
        x = x + attended.reshape(x.shape[0], -1) @ self.plain["out"].t()
        h, chosen = norm(x), chosen.long()
        weights = torch.softmax(torch.gather(h @ self.router.t(), 1, chosen), -1)
        y = x
        for j in range(CHOICES):
            up, down = self.plain["up"][chosen[:, j]], self.plain["down"][chosen[:, j]]
            gate, inner = (up * h[:, None]).sum(-1).chunk(2, -1)
            y = y + weights[:, j:j + 1] * (down * (torch.nn.functional.silu(gate) * inner)[:, None]).sum(-1)
        return y


def attend_prompt(q, k, v):
    """Causal attention of a whole prompt, fp32: q [n, heads, dim]."""
    n = q.shape[0]
    k, v = (t.float().repeat_interleave(HEADS // KV_HEADS, 1).transpose(0, 1).contiguous() for t in (k, v))
    s = q.float().transpose(0, 1).contiguous() @ k.transpose(1, 2).contiguous() / math.sqrt(DIM)
    s = s.masked_fill(torch.ones((n, n), dtype=torch.bool, device=s.device).triu(1), -math.inf)
    return (torch.softmax(s, -1) @ v).transpose(0, 1).to(q.dtype)


def run(fmt: str = "fp8", prompts=(7, 150, 64, 33), steps: int = 16, seed: int = 0):
    """The prompts in one step, then `steps` tokens of every sequence.  Returns
    (outputs [steps, batch, width], the fp32 layer's outputs of the same inputs)."""
    layer = Layer(seed)
    batch = len(prompts)
    most = -(-(max(prompts) + steps) // PAGE)
    cache = mpq.MXCache.empty(batch * most, PAGE, KV_HEADS, DIM, fmt)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    free = torch.randperm(batch * most, generator=g, device="cuda").to(torch.int32)
    table = torch.full((batch, most), -1, dtype=torch.int32, device="cuda")
    cached, taken = (torch.zeros((m,), dtype=torch.int32, device="cuda") for m in (batch, 1))

    fresh = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    tokens = sum(prompts)
    x = torch.randn((tokens, WIDTH), generator=g, device="cuda").bfloat16()
    slots, positions, starts, cached, taken = mpq.mx_plan(cached, fresh, table, free, taken, PAGE, tokens)
    q = cache.append(*layer.qkv(x), positions, slots, layer.freqs, layer.q_weight, layer.k_weight, EPS)
    keys, values = cache.read(slots, dtype=torch.bfloat16)
    ends = starts.tolist()
    spans = [slice(a, b) for a, b in zip(ends, ends[1:])]
    layer.after(x, torch.cat([attend_prompt(q[s], keys[s], values[s]) for s in spans]))
    _, kp, vp = layer.plain_qkv(x.float(), positions)
    past = [[list(kp[s]), list(vp[s])] for s in spans]   # the fp32 layer's keys and values

    space = torch.empty((max(1, cache.attend_workspace(batch, HEADS, most)),), dtype=torch.uint8, device="cuda")
    fresh = torch.ones((batch,), dtype=torch.int32, device="cuda")
    outs, plains = [], []
    for _ in range(steps):
        x = torch.randn((batch, WIDTH), generator=g, device="cuda").bfloat16()
        slots, positions, _, cached, taken = mpq.mx_plan(cached, fresh, table, free, taken, PAGE, batch)
        q = cache.append(*layer.qkv(x), positions, slots, layer.freqs, layer.q_weight, layer.k_weight, EPS)
        y, chosen = layer.after(x, cache.attend(q, table, cached, workspace=space))
        outs.append(y)

        qp, kp, vp = layer.plain_qkv(x.float(), positions)
        attended = []
        for b in range(batch):
            past[b][0].append(kp[b])
            past[b][1].append(vp[b])
            ks, vs = (torch.stack(t).repeat_interleave(HEADS // KV_HEADS, 1) for t in past[b])
            p = torch.softmax((ks * qp[b]).sum(-1) / math.sqrt(DIM), 0)
            attended.append((p[..., None] * vs).sum(0))
        plains.append(layer.plain_after(x.float(), torch.stack(attended), chosen))
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
