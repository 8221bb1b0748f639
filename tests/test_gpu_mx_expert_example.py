"""The decoder layer of examples/mx_expert_decoder.py: its decoding steps through
the library stay near the fp32 layer's.

Bound.  As for the layer without experts (tests/test_gpu_mx_example.py): a
quantization to fp4 errs by about 0.15 of a normal activation's norm, a branch of
two in turn by 0.15 sqrt(2) to 0.3, and the branches make less than half of the
output's norm.  The choices of experts are the same on both sides, and their
weights follow logits of the same kind.  A wrong page, position, expert or place
gives errors of the order of 1."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_expert_layer_stays_near_fp32(fmt):
    import torch
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    spec = importlib.util.spec_from_file_location("mx_expert_decoder", os.path.join(ROOT, "examples", "mx_expert_decoder.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    got, want = ex.run(fmt, prompts=(5, 70, 33), steps=4)
    torch.cuda.synchronize()
    err = (got - want).norm(dim=-1) / want.norm(dim=-1)
    print(f"decoder with experts {fmt}: mean {err.mean():.4f} largest {err.max():.4f}", flush=True)
    assert bool(torch.isfinite(got).all()) and float(err.max()) < 0.3
