"""The decoder layer of examples/mx_decoder.py, tightly: what its cache holds and
attends over, and its steps from the same quantized numbers.

The calls of a run are recorded.  From the keys and values in the order in which
they were written, without slots, pages or table, each sequence's attention is
computed in 64 bits over the values that the formats hold (mx_ref), and must be
the library's to the bounds of test_gpu_mx.py.  A reference without the newest
token, or with another sequence's page in place of one, is off by more than ten
times those bounds: the test would see it.

The step around it is computed from the recorded attention with activations
quantized by mx_ref's formulas: what differs is the order of fp32 sums, and so a
bf16 rounding here and there (2^-9 of a value); such a rounding moves the fp4
code of one element in some hundred by a quarter of its size.  Seven roundings
to bf16 in turn stay below 2^-6 of the output's norm."""
import importlib.util
import math
import os

import numpy as np
import pytest

import mx_ref as ref
from gpu_util import say

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
E = 2.0 ** -24


def _example():
    spec = importlib.util.spec_from_file_location("mx_decoder", os.path.join(ROOT, "examples", "mx_decoder.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    return ex


def _f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def _held(x, fmt):
    c, s = ref.quantize(ref.padded(x, ref.BLOCK), fmt)
    return ref.values(c, s, fmt)[..., :x.shape[-1]]


def _attended(q, k, v, scale):
    """(o, lse, bound) of one query head of bf16."""
    o, lse, mag = ref.attend(q, k, v, scale)
    s = np.abs(k @ q) * scale
    delta = E * ((3 * len(q) + 8) * scale * (np.abs(k) @ np.abs(q)) + 4 * (s + s.max())).max() + 2.0 ** -22
    return o, (2 * delta + 2.0 ** -16 + 2 * (len(k) + 64) * E) * mag + 2.0 ** -8 * np.abs(o)


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_decoder_steps_from_the_held_numbers(fmt, monkeypatch):
    import torch
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    ex = _example()
    say(f"case decoder layer {fmt}")
    prompts, steps = (5, 70, 33), 4
    written, read, attended = [], [], []
    plain_write, plain_read, plain_attend = ex.mpq.MXCache.write, ex.mpq.MXCache.read, ex.mpq.MXCache.attend

    def write(self, K, V, slots, **kw):
        written.append((_f64(K), _f64(V)))
        return plain_write(self, K, V, slots, **kw)

    def read_(self, slots, **kw):
        out = plain_read(self, slots, **kw)
        read.append(tuple(_f64(t) for t in out))
        return out

    def attend(self, Q, table, lengths, **kw):
        out = plain_attend(self, Q, table, lengths, **kw)
        attended.append((_f64(Q), lengths.tolist(), out.clone()))
        return out

    monkeypatch.setattr(ex.mpq.MXCache, "write", write)
    monkeypatch.setattr(ex.mpq.MXCache, "read", read_)
    monkeypatch.setattr(ex.mpq.MXCache, "attend", attend)
    inputs = []
    plain_qkv = ex.Layer.qkv

    def qkv(self, x, plain=False):
        if not plain:
            inputs.append(x.clone())
        return plain_qkv(self, x, plain)

    monkeypatch.setattr(ex.Layer, "qkv", qkv)
    got, _ = ex.run(fmt, prompts=prompts, steps=steps)
    torch.cuda.synchronize()
    batch, group, dim = len(prompts), ex.HEADS // ex.KV_HEADS, ex.DIM
    assert len(written) == batch + steps and len(read) == batch and len(attended) == steps
    assert len(inputs) == batch + steps

    # prompts: read back as held
    past = []
    for b in range(batch):
        held = [_held(t, fmt) for t in written[b]]
        past.append(held)
        for a, h in zip(read[b], held):
            assert np.array_equal(a, h)

    layer = ex.Layer(0)
    plain = {k: w.double() for k, w in layer.plain.items()}

    def linear(name, x):
        """x bf16 through the held weights, quantized by the formula."""
        q = ref.quantize(ref.padded(_f64(x), ref.ROW), "fp4")
        v = torch.from_numpy(ref.values(*q, "fp4")[:, :x.shape[1]]).cuda()
        return (v @ plain[name].t().contiguous()).bfloat16()

    for t in range(steps):
        q, lengths, out = attended[t]
        o = _f64(out)
        assert lengths == [n + t + 1 for n in prompts]
        for b in range(batch):
            for side in (0, 1):
                past[b][side] = np.concatenate([past[b][side], _held(written[batch + t][side][b:b + 1], fmt)])
        for b in range(batch):
            far = near = 0.0
            for h in range(ex.HEADS):
                k, v = (past[b][side][:, h // group] for side in (0, 1))
                want, room = _attended(q[b, h], k, v, dim ** -0.5)
                near = max(near, (np.abs(o[b, h] - want) / room).max())
                # planted in the reference: the newest token lost
                lost, _ = _attended(q[b, h], k[:-1], v[:-1], dim ** -0.5)
                far = max(far, (np.abs(o[b, h] - lost) / room).max())
            assert near <= 1 and far > 10, (t, b, near, far)
            # a page of another sequence in place of the second one
            if lengths[b] > 2 * ex.PAGE:
                k, v = (past[b][side][:, 0].copy() for side in (0, 1))
                other = past[2 if b != 2 else 1]
                for mine, theirs in ((k, other[0]), (v, other[1])):
                    mine[ex.PAGE:2 * ex.PAGE] = theirs[:ex.PAGE, 0]
                wrong, room = _attended(q[b, 0], k, v, dim ** -0.5)
                assert (np.abs(o[b, 0] - wrong) / room).max() > 10
        # the step around it
        x = inputs[batch + t]
        y = x + linear("out", out.reshape(batch, -1))
        gate, up = linear("up", ex.norm(y)).chunk(2, -1)
        y = y + linear("down", (torch.nn.functional.silu(gate.float()) * up.float()).bfloat16())
        err = (got[t] - y.float()).norm(dim=-1) / y.float().norm(dim=-1)
        assert float(err.max()) < 2.0 ** -6, err
        mine = linear("qkv", ex.norm(x)).reshape(batch, -1, dim)[:, :ex.HEADS]
        diff = torch.from_numpy(q).cuda() - mine.double()
        assert float(diff.norm() / mine.double().norm()) < 2.0 ** -6
    assert math.isfinite(float(got.sum()))
