"""What the binding of the microscaled calls does before it calls the library."""
import torch

from paper_2002_09049_amd import mpq


def test_workspace_lies_on_the_device_of_the_tensors():
    """Not on the current device, which may be another."""
    like = torch.empty((3, 5), dtype=torch.bfloat16, device="meta")
    _, n, own = mpq._space(None, lambda: 96, None, like)
    assert n == 96 and own.device == like.device and own.dtype == torch.uint8 and own.numel() == 96
    assert mpq._space(None, lambda: 0, None, like) == (None, 0, None)
    # on a stream of the caller's the library takes its own scratch
    assert mpq._space(None, lambda: 96, object(), like) == (None, 0, None)
