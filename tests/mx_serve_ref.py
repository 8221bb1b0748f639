"""Plain 64-bit implementation of a serving step's operators (numpy, from the
definitions in include/mpq.h), for the parity tests."""
from __future__ import annotations

import numpy as np

E = 2.0 ** -24
INT_MAX = 2 ** 31 - 1


def plan(cached, fresh, table, free, taken, page, max_tokens):
    """(slots, positions, starts, lengths, taken, table), one token at a time."""
    cached, fresh = np.maximum(np.asarray(cached, np.int64), 0), np.maximum(np.asarray(fresh, np.int64), 0)
    table = np.array(table)
    columns = table.shape[1]
    slots, positions = np.full(max_tokens, -1, np.int64), np.zeros(max_tokens, np.int32)
    starts, lengths, at, given = [], [], 0, int(taken)
    for b, (c, f) in enumerate(zip(cached, fresh)):
        f = min(f, max_tokens - at)
        starts.append(at)
        lengths.append(min(c + f, INT_MAX))
        held = -(-c // page)
        for j in range(held, min(-(-(c + f) // page), columns)):
            table[b, j] = free[given] if 0 <= given < len(free) else -1
            given += 1
        for i in range(f):
            p = c + i
            entry = table[b, p // page] if p // page < columns else -1
            slots[at] = entry * page + p % page if entry >= 0 else -1
            positions[at] = min(p, INT_MAX)
            at += 1
    return slots, positions, np.array(starts + [at]), np.array(lengths), given, table


def turned(x, positions, freqs, weight, eps, interleaved):
    """Heads x [n, heads, dim] fp64 turned, and the bound of a 32-bit result's
    error in units of 2^-24 (all but the rounding to the output's type).

    The inverse root errs by at most 12 units: 9 + 5 roundings in the sum of
    squares (8 in a lane, 5 between lanes), halved by the root, and the mean's,
    eps', the root's and the inverse's; the two products after it by 2, sine and
    cosine by 4 (2 of the function, the argument's and the correction's), the
    turn's products and sum by 2 of each term: at most 20 (|a| + |b|)."""
    x = np.asarray(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    half = len(freqs)
    angle = (np.asarray(positions, np.float64)[:, None] * np.asarray(freqs, np.float64))[:, None]
    first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y, size = x.copy(), np.abs(x)
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)
    size[..., first] = size[..., second] = np.abs(a) + np.abs(b)
    return y, 20 * size


def route(logits, k, renorm):
    """(chosen, weights, order, place, offsets) of fp64 logits [n, experts]."""
    x = np.where(np.isnan(logits), -np.inf, np.asarray(logits, np.float64))
    n, experts = x.shape
    chosen = np.argsort(-x, axis=1, kind="stable")[:, :k]
    top = x.max(1, keepdims=True) if n else x[:, :1]
    with np.errstate(invalid="ignore"):
        p = np.where(top == -np.inf, 0.0, np.where(x == top, 1.0, np.exp(x - top)))
    w = np.take_along_axis(p, chosen, 1)
    total = (w if renorm else p).sum(1, keepdims=True)
    w = np.where(total > 0, w / np.where(total > 0, total, 1), 0.0)
    flat = chosen.reshape(-1)
    order = np.argsort(flat, kind="stable")
    place = np.empty_like(order)
    place[order] = np.arange(len(order))
    offsets = np.searchsorted(flat[order], np.arange(experts + 1))
    return chosen, w, order, place.reshape(n, k), offsets


def groups(offsets, m):
    """The experts' (begin, end) for any content of offsets."""
    b = np.minimum(np.maximum(np.maximum.accumulate(np.asarray(offsets, np.int64)), 0), m)
    return list(zip(b[:-1], b[1:]))
