"""The microscaled operators on the paths that a call takes by its size, stream
or workspace, beside the values themselves (test_gpu_mx.py)."""
import numpy as np
import pytest

from gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    from paper_2002_09049_amd import mpq
    mpq.load()
    yield


def _uneven(shape, seed):
    """Values whose blocks are of very different sizes, so that a sum of their
    products depends on its order."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(shape, generator=g, device="cuda")
    size = torch.randint(-12, 13, (shape[0], -(-shape[1] // 32)), generator=g, device="cuda")
    return torch.ldexp(x, size.repeat_interleave(32, 1)[:, :shape[1]])


# tokens that the linear call quantizes inside the product, and rows of W from
# few to a vocabulary's
@pytest.mark.parametrize("n", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("c,d", [(40, 700), (4096, 4096), (16384, 4096), (32000, 512), (32005, 530), (65536, 4096)])
def test_linear_is_the_two_calls_bit_for_bit(n, c, d):
    import torch
    from paper_2002_09049_amd import mpq
    say(f"case mx linear against quantize and product n={n} c={c} d={d}")
    W = mpq.mx_quantize(_uneven((c, d), c + d))
    X = _uneven((n, d), n)
    two = mpq.mx_product(*mpq.mx_quantize(X), *W, d)
    one = mpq.mx_linear(X, *W)
    assert bool(torch.isfinite(one).all())
    assert torch.equal(one, two), int((one != two).sum())
