"""The product's kernels for many tokens: 16-bit outputs, every tile with K
longer than its ring, and tokens or rows of W one past a tile.  References and
bounds as in test_gpu_mx.py: products of fp4 values are exact, the sum has at
most 128 + stages + 16 roundings of 2^-24 of sum |x w|, the output one."""
import pytest

from gpu_util import say

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    from paper_2002_09049_amd import mpq
    mpq.load()
    yield


def _dt(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


# n, c, d, tile: each past its ring of four stages of 128 and past one scale load (2048)
CASES = [(500, 4001, 2200, "2,1"), (1000, 4001, 2300, "2,2"), (2000, 4001, 2500, "4,2"), (3900, 4001, 2600, "4,4"),
         (129, 4097, 5000, "2,1"), (1025, 4096, 1152, "4,2"), (2049, 3585, 640, "4,2"), (4097, 4096, 2176, "4,4")]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("n,c,d,tile", CASES)
def test_tiles_by_type(n, c, d, tile, dtype):
    import torch
    from paper_2002_09049_amd import mpq
    say(f"case mx tiles n={n} c={c} d={d} {dtype}")
    g = torch.Generator(device="cuda").manual_seed(n + d)
    X = torch.randn((n, d), generator=g, device="cuda") * torch.exp(torch.randn((d,), generator=g, device="cuda"))
    W = torch.randn((c, d), generator=g, device="cuda") / d ** 0.5
    X = X.to(_dt(dtype))
    b = torch.randn((c,), generator=g, device="cuda")
    w = mpq.mx_quantize(W)
    room = torch.full((n, c + 6), -7.0, dtype=_dt(dtype), device="cuda")     # rows apart, not aligned to vectors
    mpq.timing_enable(True)
    try:
        Y = mpq.mx_linear(X, *w, bias=b, out=room[:, 3:c + 3])
        names = [k for k, _ in mpq.timing_read()]
    finally:
        mpq.timing_enable(False)
    assert names == ["mx_quantize_kernel", f"mx_tile_kernel<{tile}>"]
    assert bool((room[:, :3] == -7).all()) and bool((room[:, c + 3:] == -7).all())
    # contiguous rows give the same bits
    assert torch.equal(mpq.mx_linear(X, *w, bias=b), Y)
    x, v = mpq.mx_dequantize(*mpq.mx_quantize(X), d).double(), mpq.mx_dequantize(*w, d).double().t().contiguous()
    want = x @ v + b.double()
    mag = x.abs() @ v.abs() + b.double().abs()
    err = (Y.double() - want).abs()
    most = (128 + -(-d // 128) + 16) * E * mag + UNIT[dtype] * want.abs() + (2.0 ** -25 if dtype == "f16" else 0)
    assert bool((err <= most).all()), float((err / most).max())


# without a workspace a call on a stream takes the library's own scratch there
@pytest.mark.parametrize("n,c,d", [(6, 300, 700), (64, 500, 2100), (700, 1000, 1300)])
def test_scratch_on_a_stream(n, c, d):
    import torch
    from paper_2002_09049_amd import mpq
    say(f"case mx linear scratch on a stream n={n}")
    g = torch.Generator(device="cuda").manual_seed(n)
    w = mpq.mx_quantize(torch.randn((c, d), generator=g, device="cuda"))
    X = [torch.randn((n, d), generator=g, device="cuda").half() for _ in range(3)]
    want = [mpq.mx_linear(x, *w) for x in X]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = [mpq.mx_linear(x, *w, stream=side) for x in X]     # the scratch of one is the next one's
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_attend_scratch_on_a_stream():
    import torch
    from paper_2002_09049_amd import mpq
    say("case mx attend scratch on a stream")
    g = torch.Generator(device="cuda").manual_seed(4)
    cache = mpq.MXCache.empty(260, 16, 2, 64, "fp4")
    slots = torch.arange(260 * 16, device="cuda")
    cache.write(*(torch.randn((slots.numel(), 2, 64), generator=g, device="cuda") for _ in "KV"), slots)
    table = torch.randperm(260, generator=g, device="cuda").to(torch.int32).reshape(2, 130)
    length = torch.tensor([2080, 1999], dtype=torch.int32, device="cuda")
    assert cache.attend_workspace(2, 8, 130) > 0
    Q = [torch.randn((2, 8, 64), generator=g, device="cuda").bfloat16() for _ in range(3)]
    want = [cache.attend(q, table, length, with_lse=True) for q in Q]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = [cache.attend(q, table, length, with_lse=True, stream=side) for q in Q]
    side.synchronize()
    for (o, e), (a, b) in zip(got, want):
        assert torch.equal(o, a) and torch.equal(e, b)


def test_captured_calls_of_two_launches():
    """A linear call that quantizes first, by the kernels for few, some tens of
    and many tokens, and attention with its join, captured with the caller's
    workspaces and replayed over changing inputs, with eager work between."""
    import torch
    from paper_2002_09049_amd import mpq
    say("case mx captured linear and join")
    g = torch.Generator(device="cuda").manual_seed(9)
    c, d = 2000, 2048
    w = mpq.mx_quantize(torch.randn((c, d), generator=g, device="cuda"))
    tokens = (8, 64, 1500)
    X = [torch.zeros((n, d), dtype=torch.bfloat16, device="cuda") for n in tokens]
    spaces = [torch.empty((mpq.mx_linear_workspace(n, c, d),), dtype=torch.uint8, device="cuda") for n in tokens]
    cache = mpq.MXCache.empty(300, 16, 2, 64, "fp8")
    slots = torch.arange(300 * 16, device="cuda")
    cache.write(*(torch.randn((slots.numel(), 2, 64), generator=g, device="cuda") for _ in "KV"), slots)
    table = torch.randperm(300, generator=g, device="cuda").to(torch.int32).reshape(2, 150)
    lengths = torch.zeros((2,), dtype=torch.int32, device="cuda")
    Q = torch.zeros((2, 8, 64), dtype=torch.bfloat16, device="cuda")
    spaces.append(torch.empty((cache.attend_workspace(2, 8, 150),), dtype=torch.uint8, device="cuda"))
    assert min(s.numel() for s in spaces) > 0

    def step():
        return [mpq.mx_linear(x, *w, workspace=s) for x, s in zip(X, spaces)] + list(
            cache.attend(Q, table, lengths, with_lse=True, workspace=spaces[-1]))

    def set_inputs(i):
        for t in X + [Q]:
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        lengths.copy_(torch.tensor([2400 - 97 * i, 1300 * (i % 2) + 3], dtype=torch.int32))

    set_inputs(0)
    mpq.timing_enable(True)
    try:
        step()
        names = [k for k, _ in mpq.timing_read()]
    finally:
        mpq.timing_enable(False)
    assert names[1::2] == ["mx_few_kernel", "mx_slab_kernel", names[5], "mx_attend_join_kernel"]
    assert names[5].startswith("mx_tile_kernel") and names[0::2] == ["mx_quantize_kernel"] * 3 + ["mx_attend_kernel"]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for i in range(5):
        set_inputs(i)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        want = step()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b) and bool(torch.isfinite(b.float()).all()), i


# a size for each of the product's kernels
KINDS = [(1, 300, 2000), (4, 40, 700), (12, 300, 2000), (40, 500, 2100), (500, 4001, 1300), (1000, 4001, 1300),
         (2000, 4001, 1300), (3900, 4001, 700)]


@pytest.mark.parametrize("n,c,d", KINDS)
def test_blocks_of_different_sizes(n, c, d):
    """Blocks 2^24 apart within a row: small ones beside large ones err by
    roundings of the whole sum alone."""
    import torch
    from paper_2002_09049_amd import mpq
    say(f"case mx uneven blocks n={n} c={c} d={d}")
    g = torch.Generator(device="cuda").manual_seed(n + c)

    def uneven(r):
        x = torch.randn((r, d), generator=g, device="cuda")
        size = torch.randint(-12, 13, (r, -(-d // 32)), generator=g, device="cuda")
        return torch.ldexp(x, size.repeat_interleave(32, 1)[:, :d])

    w, x = mpq.mx_quantize(uneven(c)), uneven(n)
    Y = mpq.mx_linear(x, *w)
    xv, wv = mpq.mx_dequantize(*mpq.mx_quantize(x), d).double(), mpq.mx_dequantize(*w, d).double().t().contiguous()
    want, mag = xv @ wv, xv.abs() @ wv.abs()
    most = (128 + -(-d // 128) + 16) * E * mag + E * want.abs()
    err = (Y.double() - want).abs()
    assert bool((err <= most).all()), float((err / most).max())
