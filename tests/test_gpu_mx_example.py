"""The decoder layer of examples/mx_decoder.py: its decoding steps through the
library stay near the fp32 layer's.

Bound.  fp4 rounds an element to one mantissa bit: a relative error of up to
1/4, uniform within it about 0.11 rms of the large elements, and about 0.15 of a
normal activation's norm with the smaller ones.  The layer's output is its input
(exact, bf16) plus two branches whose matrices are held exactly in both
computations; each branch passes two quantizations in turn (0.15 each, and
the attention's keys and values), so a branch errs by about 0.15 sqrt(2) to 0.3,
and the sum, a third to a half of whose norm the branches make, by less than
0.3.  A wrong page, head or scale gives errors of the order of 1."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_decoder_layer_stays_near_fp32(fmt):
    import torch
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    spec = importlib.util.spec_from_file_location("mx_decoder", os.path.join(ROOT, "examples", "mx_decoder.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    got, want = ex.run(fmt, prompts=(5, 70, 33), steps=4)
    torch.cuda.synchronize()
    err = (got - want).norm(dim=-1) / want.norm(dim=-1)
    print(f"decoder {fmt}: mean {err.mean():.4f} largest {err.max():.4f}", flush=True)
    assert bool(torch.isfinite(got).all()) and float(err.max()) < 0.3
