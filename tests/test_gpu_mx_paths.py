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


def _pool_of(t):
    """The stream whose pool of torch's allocator a tensor's memory belongs to."""
    import torch
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not of the allocator")


def test_outputs_belong_to_the_stream_that_writes_them():
    """With stream=, a call's new outputs come from that stream's pool: memory
    that the current stream's work may still use is not among it."""
    import torch
    from paper_2002_09049_amd import mpq
    say("case outputs on a stream")
    W, X = _uneven((48, 96), 1), _uneven((6, 96), 2)
    batch = X.t().contiguous()
    ints = torch.randint(-100, 101, (5, 96), device="cuda").to(torch.int8)
    cache = mpq.MXCache.empty(9, 16, 2, 64, "fp8")
    K, V = _uneven((20, 128), 3).reshape(20, 2, 64), _uneven((20, 128), 4).reshape(20, 2, 64)
    slots = torch.arange(20, device="cuda")
    table = torch.arange(2, dtype=torch.int32, device="cuda")[None]
    length = torch.tensor([20], dtype=torch.int32, device="cuda")
    codes, scales = mpq.mx_quantize(W)
    xc, xs = mpq.mx_quantize(X)
    fit = mpq.fit_layer(W, 4, 3, 64, 0.01)
    A, _ = mpq.integer_scales(fit[1], fit[2], 8)
    cache.write(K, V, slots)

    def calls(stream):
        yield "fit_layer", mpq.fit_layer(W, 4, 3, 64, 0.01, stream=stream)
        yield "fit_layer_calib", mpq.fit_layer_calib(W, 4, 3, 64, batch, 0.01, stream=stream)
        yield "output_error", mpq.output_error(W, *fit[:3], batch, with_ref=True, stream=stream)
        yield "reconstruct", (mpq.reconstruct(*fit[:3], stream=stream),)
        yield "integer_scales", mpq.integer_scales(fit[1], fit[2], 8, stream=stream)
        yield "integer_forward", (mpq.integer_forward(fit[0], A, fit[2], ints, 8, stream=stream),)
        yield "mx_quantize", mpq.mx_quantize(W, stream=stream)
        yield "mx_dequantize", (mpq.mx_dequantize(codes, scales, 96, stream=stream),)
        yield "mx_product", (mpq.mx_product(xc, xs, codes, scales, 96, stream=stream),)
        yield "mx_linear", (mpq.mx_linear(X, codes, scales, stream=stream),)
        yield "read", cache.read(slots, stream=stream)
        yield "attend", cache.attend(K[:1], table, length, with_lse=True, stream=stream)

    want = dict(calls(None))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, torch.cuda.ExternalStream(side.cuda_stream)):
        for name, got in calls(stream):
            side.synchronize()
            for a, b in zip(got, want[name]):
                assert _pool_of(a) == side.cuda_stream, name
                assert torch.equal(a, b), name


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_attend_queries_up_to_the_largest_fp32(fmt):
    """fp32 queries past bf16's largest value are finite, and split exactly; an
    infinity or a NaN gives its own head a NaN and no other."""
    import torch
    import mx_ref as ref
    from paper_2002_09049_amd import mpq
    say(f"case mx attend huge queries {fmt}")
    rng = np.random.default_rng(6)
    n, dim = 50, 64
    cache = mpq.MXCache.empty(4, 16, 1, dim, fmt)
    K = (rng.standard_normal((n, 1, dim)) * 2.0 ** -110).astype(np.float32)
    V = rng.standard_normal((n, 1, dim)).astype(np.float32)
    slots = torch.arange(n, device="cuda")
    cache.write(torch.from_numpy(K).cuda(), torch.from_numpy(V).cuda(), slots)
    k, v = (t.double().cpu().numpy()[:, 0] for t in cache.read(slots))
    q = (rng.uniform(-1, 1, (1, 5, dim)) * 2.0 ** 126).astype(np.float32)
    top = np.finfo(np.float32).max
    q[0, 0, ::5], q[0, 1, ::7], q[0, 2, 3] = top, -top, np.float32(3.3961e38)   # bf16: 3.38953e38, ties at 3.39618e38
    q[0, 3, 9], q[0, 4, 60] = np.inf, np.nan
    scale = 2.0 ** -19
    table = torch.arange(4, dtype=torch.int32, device="cuda")[None]
    O, lse = cache.attend(torch.from_numpy(q).cuda(), table, torch.tensor([n], dtype=torch.int32, device="cuda"),
                          scale=scale, with_lse=True)
    O, lse = O.double().cpu().numpy()[0], lse.double().cpu().numpy()[0]
    assert np.isnan(O[3:]).all() and np.isnan(lse[3:]).all()
    e = 2.0 ** -24
    for h in range(3):
        x = q[0, h].astype(np.float64)
        want, l, mag = ref.attend(x, k, v, scale)
        s = np.abs(k @ x) * scale
        delta = e * ((3 * dim + 8) * scale * (np.abs(k) @ np.abs(x)) + 4 * (s + s.max())).max() + 2.0 ** -22
        assert (np.abs(O[h] - want) <= (2 * delta + e + 2 * (n + 64) * e) * mag + e * np.abs(want)).all()
        assert abs(lse[h] - l) <= delta + (n + 64) * e + 2.0 ** -22 * (1 + abs(l))


def test_a_workspace_that_is_too_small_is_refused():
    """An empty one too, which has no address; where none is needed, it will do."""
    import torch
    from paper_2002_09049_amd import mpq
    say("case mx small workspaces")
    empty = torch.empty((0,), dtype=torch.uint8, device="cuda")
    W = mpq.mx_quantize(_uneven((48, 96), 1))
    need = mpq.mx_linear_workspace(6, 48, 96)
    assert need > 0 and mpq.mx_linear_workspace(3, 48, 96) == 0
    X = _uneven((6, 96), 2)
    for space in (empty, torch.empty((need - 1,), dtype=torch.uint8, device="cuda")):
        with pytest.raises(mpq.MPQError, match="too small"):
            mpq.mx_linear(X, *W, workspace=space)
    assert torch.equal(mpq.mx_linear(X[:3], *W, workspace=empty), mpq.mx_linear(X[:3], *W))
    cache = mpq.MXCache.empty(200, 16, 1, 32, "fp8")
    Q = _uneven((1, 32), 3)[:, None]
    table = torch.arange(200, dtype=torch.int32, device="cuda")[None]
    length = torch.tensor([30], dtype=torch.int32, device="cuda")
    assert cache.attend_workspace(1, 1, 200) > 0 and cache.attend_workspace(1, 1, 2) == 0
    with pytest.raises(mpq.MPQError, match="too small"):
        cache.attend(Q, table, length, workspace=empty)
    assert torch.equal(cache.attend(Q, table[:, :2], length, workspace=empty), cache.attend(Q, table[:, :2], length))


def _room(gib):
    import torch
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB of device memory")


def test_rows_past_one_launch_dimension():
    """2^35 held elements and more: 2^24 workgroups of 256 threads, whose
    threads no longer count in 32 bits."""
    import torch
    from paper_2002_09049_amd import mpq
    _room(24)
    rows = (1 << 28) + 37
    say(f"case mx rows {rows} x 1")
    some = torch.tensor([1.0, -1.5, 0.0, 2.0, -3.0, 0.75, 4.0, -6.0, 0.5, 12.0, -0.0625], device="cuda").half()
    X = some[torch.arange(rows, dtype=torch.int32, device="cuda") % 11][:, None]      # each held exactly
    codes, scales = mpq.mx_quantize(X)
    Y = mpq.mx_dequantize(codes, scales, 1, dtype=torch.float16)
    assert torch.equal(X, Y)
    tail = mpq.mx_quantize(X[-50:])
    assert torch.equal(codes[-50:], tail[0]) and torch.equal(scales[-50:], tail[1])


@pytest.mark.parametrize("n", [1, 6])
def test_products_past_one_launch_dimension(n):
    """2^27 rows of W and more: 2^23 workgroups of 512 threads."""
    import torch
    from paper_2002_09049_amd import mpq
    _room(30)
    c, d, part = (1 << 27) + 4099, 40, 4096
    say(f"case mx product of {c} rows, {n} tokens")
    w = mpq.mx_quantize(_uneven((part, d), 5))
    codes, scales = (torch.empty((c, t.shape[1]), dtype=torch.uint8, device="cuda") for t in w)
    for whole, t in ((codes, w[0]), (scales, w[1])):
        whole[:c // part * part].view(-1, part, t.shape[1])[:] = t
        whole[c // part * part:] = t[:c % part]
    X = _uneven((n, d), 6)
    few = mpq.mx_linear(X, *w)
    for Y in (mpq.mx_linear(X, codes, scales), mpq.mx_product(*mpq.mx_quantize(X), codes, scales, d)):
        assert torch.equal(Y[:, :c // part * part].view(n, -1, part), few[:, None].expand(n, c // part, part))
        assert torch.equal(Y[:, c // part * part:], few[:, :c % part])


def test_cache_past_one_launch_dimension():
    """2^30 rows of one block and more, of which a few have a slot."""
    import torch
    from paper_2002_09049_amd import mpq
    _room(40)
    n, page = (1 << 30) + 70, 16
    say(f"case mx cache of {n} tokens")
    cache = mpq.MXCache.empty(8, page, 1, 1, "fp8")
    K = torch.zeros((n, 1, 1), dtype=torch.bfloat16, device="cuda")
    slots = torch.full((n,), -1, dtype=torch.int64, device="cuda")
    where = torch.tensor([0, 5, (1 << 20) * 64 - 1, (1 << 20) * 64, (1 << 30) - 1, 1 << 30, n - 1], device="cuda")
    value = torch.tensor([1.0, -2.0, 0.5, 3.0, -4.0, 1.5, 7.0], device="cuda").bfloat16()     # held exactly
    K[where, 0, 0] = value
    slots[where] = torch.arange(7, device="cuda") * 17
    cache.write(K, K, slots)
    k, v = cache.read(slots[where], dtype=torch.bfloat16)
    assert torch.equal(k[:, 0, 0], value) and torch.equal(v[:, 0, 0], value)
    k, v = cache.read(slots, dtype=torch.bfloat16)
    assert torch.equal(k, K) and torch.equal(v, K)


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("small", ["keys", "values"])
def test_attend_smallest_blocks(fmt, small):
    """Blocks of the least scale bytes: fp4 exactly, fp8 with each element
    rounded to a multiple of 2^-133 (at most 2^-134 off)."""
    import torch
    import mx_ref as ref
    from paper_2002_09049_amd import mpq
    say(f"case mx attend smallest blocks {fmt} {small}")
    n, dim, e, least = 90, 64, 2.0 ** -24, 2.0 ** -134 if fmt == "fp8" else 0.0
    for power in (-114, -117, -119, -122, -125, -127):
        rng = np.random.default_rng(-power)
        cache = mpq.MXCache.empty(6, 16, 1, dim, fmt)
        K, V = (rng.standard_normal((n, 1, dim)).astype(np.float32) for _ in "KV")
        q = rng.uniform(-1, 1, (1, 1, dim))
        scale = dim ** -0.5
        if small == "keys":
            K = np.ldexp(K, power)
            q, scale = np.ldexp(q, 120), scale * 2.0 ** (-power - 120)
        else:
            V = np.ldexp(V, power)
        q = q.astype(np.float32)
        slots = torch.arange(n, device="cuda")
        cache.write(torch.from_numpy(K).cuda(), torch.from_numpy(V).cuda(), slots)
        k, v = (t.double().cpu().numpy()[:, 0] for t in cache.read(slots))
        table = torch.arange(6, dtype=torch.int32, device="cuda")[None]
        O, lse = cache.attend(torch.from_numpy(q).cuda(), table, torch.tensor([n], dtype=torch.int32, device="cuda"),
                              scale=scale, with_lse=True)
        x = q[0, 0].astype(np.float64)
        want, l, mag = ref.attend(x, k, v, scale)
        s = np.abs(k @ x) * scale
        delta = e * ((3 * dim + 8) * scale * (np.abs(k) @ np.abs(x)) + 4 * (s + s.max())).max() + 2.0 ** -22
        if small == "keys":
            delta += scale * least * np.abs(x).sum()
        room = (2 * delta + e + 2 * (n + 64) * e) * mag + e * np.abs(want) + 2.0 ** -149 * (n + 64)
        if small == "values":
            room += least
        o = O.double().cpu().numpy()[0, 0]
        assert (np.abs(o - want) <= room).all(), (power, np.max(np.abs(o - want) / room))
        assert abs(float(lse) - l) <= delta + (n + 64) * e + 2.0 ** -22 * (1 + abs(l)), power
