"""Fits of very many channels: several layers go in launches of at most 2^22
channels, and a layer whose launch would have 2^32 threads is refused."""
import pytest

from gpu_util import say

pytestmark = pytest.mark.gpu


def _room(gib):
    import torch
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB of device memory")


def test_layers_of_many_channels():
    import torch
    from paper_2002_09049_amd import mpq
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    _room(12)
    g = torch.Generator(device="cuda").manual_seed(1)
    W = [torch.randn((c, d), generator=g, device="cuda") for c, d in ((3 << 20, 17), (2 << 20, 20), ((1 << 20) + 7, 17),
                                                                      (5 << 20, 4), (100, 18))]
    say("case fit of layers of 11 M channels")
    s = mpq.LayerSet(W, 2)
    s.fit(3, 16, 0.01)
    for i, w in enumerate(W):
        for a, b in zip(mpq.fit_layer(w, 3, 2, 16, 0.01), (s.codes[i], s.scales[i], s.counts[i], s.fit_err[i])):
            assert torch.equal(a, b), i


def test_a_layer_past_one_launch_is_refused():
    import torch
    from paper_2002_09049_amd import mpq
    _room(24)
    say("case fit of 2^26 channels")
    W = torch.ones(((1 << 26) + 3, 17), device="cuda")    # one wavefront a channel
    with pytest.raises(mpq.MPQError, match="invalid argument"):
        mpq.fit_layer(W, 2, 1, 4, 0.0, with_err=False)
    codes, scales, counts, _ = mpq.fit_layer(W[:1 << 20], 2, 1, 4, 0.0, with_err=False)
    assert bool((counts == 1).all()) and bool((codes == 1).all())
