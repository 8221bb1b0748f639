"""A serving step's operators (mpq_mx_plan, _rotate, _cache_append, _route,
_experts, _combine) through the binding against the plain 64-bit implementation
of mx_serve_ref: whole numbers equal, the cache's bytes those of heads turned and
quantized in 64 bits, other values within bounds that follow from fp32 sums.

Bounds, with u = 2^-24 and h half a step of the output's type (relative):
  turned heads  mx_serve_ref.turned's units, and h |y|.
  weights       a logit's difference from the top is rounded once (u |v - top|),
                exp errs by 2 units, sums of n parts by their depth (experts / 64 +
                6), the quotient by 1; numerator and denominator alike.
  products      (128 + steps + 16) u sum |x w| as in test_gpu_mx.py, and h |y|.
  sums          (k + 1) u of the terms' magnitudes, and h |z|.
A value below the type's smallest normal number is off by half of the spacing
there."""
import numpy as np
import pytest

import mx_ref
import mx_serve_ref as ref
from gpu_util import say

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}
TYPES = ["f32", "f16", "bf16"]


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


def _dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _f64(t):
    return t.double().cpu().numpy()


def _near(got, want, bound, dtype, what=""):
    got = _f64(got)
    limit = bound + HALF[dtype] * np.abs(want) + TINY[dtype]
    bad = ~(np.abs(got - want) <= limit)
    assert not bad.any(), (what, np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], np.broadcast_to(limit, want.shape)[bad][:5])


def _activations(rng, shape):
    x = rng.standard_normal(shape) * np.exp(rng.standard_normal(shape[-1]))
    x[rng.random(shape) < 0.02] = 0.0
    return x


# ---------------------------------------------------------------- plan


def _requests(rng, batch, most, page):
    cached = rng.integers(0, most, batch)
    fresh = np.where(rng.random(batch) < 0.3, rng.integers(0, most, batch), rng.integers(0, 2, batch))
    cached[rng.random(batch) < 0.2] = 0
    edge = rng.random(batch) < 0.2
    cached[edge] = cached[edge] // page * page
    return cached.astype(np.int32), fresh.astype(np.int32)


def _planned(cached, fresh, table, free, taken, page, tokens, ld=None, stream=None):
    import torch
    from paper_2002_09049_amd import mpq
    wide = _dev(np.full((table.shape[0], ld or table.shape[1]), -7, np.int32))
    wide[:, :table.shape[1]] = _dev(table)
    view = wide[:, :table.shape[1]]
    out = mpq.mx_plan(_dev(cached), _dev(fresh), view, _dev(free), _dev(np.array([taken], np.int32)), page, tokens, stream=stream)
    torch.cuda.synchronize()
    assert (wide[:, table.shape[1]:].cpu().numpy() == -7).all()
    return [t.cpu().numpy() for t in out] + [view.cpu().numpy()]


def _same_plan(got, want):
    for g, w, name in zip(got, want, ("slots", "positions", "starts", "lengths", "taken", "table")):
        assert np.array_equal(g.reshape(-1), np.reshape(w, -1)), name


@pytest.mark.parametrize("batch,most,page,extra,ld", [
    (1, 2, 16, 0, None), (1, 1, 16, 5, None), (3, 70, 16, 0, 9), (64, 500, 48, 3, None), (256, 90, 64, 0, 31), (257, 90, 16, 700, None),
    (1023, 40, 32, 0, None), (1025, 40, 16, 1, None), (2500, 20, 16, 9, None), (2, 70000, 65536, 4, None), (5, 4000, 256, 0, None)])
def test_plan(batch, most, page, extra, ld):
    rng = np.random.default_rng(batch * 1000 + most)
    for short in (False, True):
        cached, fresh = _requests(rng, batch, most, page)
        need = -(-(cached + fresh) // page)
        held = -(-cached // page)
        columns = max(1, int(need.max()) - (1 if short else 0)) + (0 if short else 2)
        if ld is not None:
            columns = min(columns, ld)
        table = np.full((batch, columns), -1, np.int32)
        pages = rng.permutation(int(held.sum() + (need - held).sum()) + 5).astype(np.int32)
        at = 0
        for b in range(batch):
            n = min(held[b], columns)
            table[b, :n] = pages[at:at + n]
            at += n
        free = pages[at:]
        if short:
            free = free[:max(2, len(free) // 2)]
        total = int(fresh.sum())
        tokens = max(0, total - total // 3) if short else total + extra
        want = ref.plan(cached, fresh, table, free, 2, page, tokens)
        _same_plan(_planned(cached, fresh, table, free, 2, page, tokens, ld), want)


def test_plan_edges():
    """No sequences, no tokens, no columns, no free pages, entries and counts below
    zero, more tokens than rows, lengths at the end of int32."""
    i = np.array
    for case in [
        (i([], np.int32), i([], np.int32), np.zeros((0, 3), np.int32), i([4], np.int32), 0, 16, 5),
        (i([3, 0], np.int32), i([0, 0], np.int32), np.full((2, 2), -1, np.int32), i([4], np.int32), 0, 16, 0),
        (i([3, 0], np.int32), i([2, 9], np.int32), np.full((2, 2), -1, np.int32), i([], np.int32), 0, 16, 12),
        (i([-5, 17], np.int32), i([-1, 40], np.int32), i([[5, 6], [2, -4]], np.int32), i([8, 9, 1], np.int32), 1, 16, 41),
        (i([0] * 9, np.int32), i([30] * 9, np.int32), np.full((9, 4), -1, np.int32), np.arange(40, dtype=np.int32), 0, 16, 100),
        (i([2 ** 31 - 1, 2 ** 31 - 20], np.int32), i([5, 30], np.int32), np.full((2, 4), 3, np.int32), i([1], np.int32), 0, 16, 40),
        (i([0], np.int32), i([20], np.int32), np.full((1, 4), -1, np.int32), np.arange(4, dtype=np.int32), -1, 16, 20),
        (i([1, 1], np.int32), i([2 ** 31 - 1] * 2, np.int32), np.full((2, 4), -1, np.int32), np.arange(9, dtype=np.int32), 0, 16, 70),
    ]:
        _same_plan(_planned(*case), ref.plan(*case))
    from paper_2002_09049_amd import mpq
    a = _dev(np.array([3], np.int32))
    out = mpq.mx_plan(a, a, _dev(np.zeros((1, 0), np.int32)), a, a, 16, 4)
    assert out[0].tolist() == [-1] * 4 and out[1].tolist() == [3, 4, 5, 0] and out[4].tolist() == [3]


# ---------------------------------------------------------------- rotate


def _heads(rng, n, heads, dim, dtype, layout):
    """Heads on the device, as a view of a wider tensor for layout 1, of a
    transposed one for layout 2."""
    import torch
    x = _dev(_activations(rng, (n, heads, dim)), _dt(dtype))
    if layout == 1:
        wide = torch.zeros((n, heads + 3, dim + 5), dtype=x.dtype, device="cuda")
        wide[:, 2:2 + heads, 3:3 + dim] = x
        return wide[:, 2:2 + heads, 3:3 + dim]
    if layout == 2:
        return x.transpose(0, 1).contiguous().transpose(0, 1)
    return x


def _freqs(rot, theta=10000.0):
    return theta ** (-2.0 * np.arange(rot // 2) / max(rot, 1))


SHAPES = [(1, 1, 1, 1, 0), (1, 32, 8, 128, 128), (3, 2, 1, 2, 2), (5, 7, 1, 80, 40), (4, 3, 3, 33, 10), (9, 4, 2, 64, 64),
          (17, 5, 5, 40, 20), (2, 6, 3, 256, 256), (33, 2, 2, 192, 96), (130, 8, 2, 96, 96), (7, 3, 1, 255, 254), (4, 2, 2, 8, 6),
          # several tokens a wavefront
          (4099, 2, 1, 128, 128), (4097, 3, 1, 80, 40), (4110, 1, 1, 256, 256), (4101, 5, 2, 30, 16), (4098, 2, 1, 64, 64)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,heads,kv,dim,rot", SHAPES)
def test_rotate(n, heads, kv, dim, rot, dtype):
    import torch
    from paper_2002_09049_amd import mpq
    rng = np.random.default_rng(n * 7 + dim)
    for interleaved in (False, True):
        for layout, (qn, kn), far in ((0, (True, True), 0), (1, (False, True), 2 ** 20), (2, (True, False), -3), (0, (False, False), 2 ** 31 - 9 - n)):
            Q, K = _heads(rng, n, heads, dim, dtype, layout), _heads(rng, n, kv, dim, dtype, layout)
            positions = (np.arange(n) + far).astype(np.int32)
            freqs = _freqs(rot)
            qw, kw = (rng.uniform(0.5, 1.5, dim).astype(np.float32) if w else None for w in (qn, kn))
            got = mpq.mx_rotate(Q, K, _dev(positions), _dev(freqs), *(None if w is None else _dev(w) for w in (qw, kw)),
                                eps=1e-5, interleaved=interleaved)
            for g, x, w in zip(got, (Q, K), (qw, kw)):
                y, units = ref.turned(_f64(x), positions, freqs, w, float(np.float32(1e-5)), interleaved)
                _near(g, y, E * units, dtype, (interleaved, layout, far))
            # into tensors of the caller's, and in place
            to = [_heads(rng, n, h, dim, dtype, 1) for h in (heads, kv)]
            mpq.mx_rotate(Q, K, _dev(positions), _dev(freqs), *(None if w is None else _dev(w) for w in (qw, kw)), eps=1e-5,
                          interleaved=interleaved, out=to)
            again = mpq.mx_rotate(Q, K, _dev(positions), _dev(freqs), *(None if w is None else _dev(w) for w in (qw, kw)),
                                  eps=1e-5, interleaved=interleaved, out=(Q, K))
            assert again[0] is Q
            for g, t, x in zip(got, to, (Q, K)):
                assert torch.equal(g, t) and torch.equal(g, x)


def test_rotate_leaves_the_rest():
    """Elements past rot are the input's bits without a norm; a head of NaN or of
    zeros has no influence on the others."""
    import torch
    from paper_2002_09049_amd import mpq
    rng = np.random.default_rng(5)
    Q, K = _heads(rng, 6, 4, 72, "bf16", 0), _heads(rng, 6, 2, 72, "bf16", 0)
    positions, freqs, w = _dev(np.arange(6, dtype=np.int32)), _dev(_freqs(24)), _dev(np.ones(72, np.float32))
    q, k = mpq.mx_rotate(Q, K, positions, freqs)
    assert torch.equal(q[..., 24:], Q[..., 24:]) and torch.equal(k[..., 24:], K[..., 24:])
    assert torch.equal(q[0], Q[0])   # position 0
    q, k = mpq.mx_rotate(Q, K, positions, freqs, w, w)
    Q2 = Q.clone()
    Q2[3, 1], Q2[4, 2, 50], Q2[2, 0] = float("nan"), float("inf"), 0.0
    q2, k2 = mpq.mx_rotate(Q2, K, positions, freqs, w, w)
    assert torch.equal(k, k2) and (q2[2, 0] == 0).all() and q2[3, 1].isnan().all()
    q2[3, 1], q2[4, 2], q2[2, 0] = q[3, 1], q[4, 2], q[2, 0]
    assert torch.equal(q, q2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("n,heads,kv,dim,rot,page", [(1, 8, 2, 128, 128, 16), (5, 7, 1, 80, 40, 48), (37, 2, 2, 33, 10, 16),
                                                     (130, 6, 3, 64, 64, 64), (20, 4, 4, 256, 128, 32), (3, 2, 1, 192, 0, 16),
                                                     (9, 5, 5, 32, 32, 16), (12, 2, 1, 256, 256, 16),
                                                     (4099, 2, 1, 128, 128, 16), (4097, 1, 2, 80, 40, 48), (4101, 3, 2, 32, 32, 16)])
def test_append(n, heads, kv, dim, rot, page, fmt, dtype):
    import torch
    from paper_2002_09049_amd import mpq
    rng = np.random.default_rng(n + dim)
    for interleaved, normed, layout in ((False, True, 0), (True, True, 1), (False, False, 2)):
        Q, K, V = (_heads(rng, n, h, dim, dtype, layout) for h in (heads, kv, kv))
        K[n // 2, 0, dim // 2] = float("inf")
        V[0, kv - 1, 0] = float("nan")
        positions, freqs = (np.arange(n) * 7919).astype(np.int32), _freqs(rot)
        w = [rng.uniform(0.5, 1.5, dim).astype(np.float32) if normed else None for _ in "qk"]
        on = [None if x is None else _dev(x) for x in w]
        pages = -(-n // page) + 2
        slots = rng.permutation(pages * page)[:n]
        if n > 1:
            slots[n // 3] = -1
        if n > 4:
            slots[4] = pages * page
        cache = mpq.MXCache.empty(pages, page, kv, dim, fmt)
        for t in cache.tensors:
            t.fill_(77)
        q = cache.append(Q, K, V, _dev(positions), _dev(slots.astype(np.int64)), _dev(freqs), *on, eps=1e-5,
                         interleaved=interleaved)
        assert torch.equal(q, mpq.mx_rotate(Q, K, _dev(positions), _dev(freqs), *on, eps=1e-5, interleaved=interleaved)[0])
        live = (slots >= 0) & (slots < pages * page)
        where, at = slots[live] // page, slots[live] % page
        with np.errstate(invalid="ignore"):
            turned, _ = ref.turned(_f64(K), positions, freqs, w[1], float(np.float32(1e-5)), interleaved)
        for x, codes, scales in ((turned, cache.tensors[0], cache.tensors[2]), (_f64(V), cache.tensors[1], cache.tensors[3])):
            c, sc = mx_ref.quantize(mx_ref.padded(x[live], 32), fmt)
            codes, scales = codes.cpu().numpy(), scales.cpu().numpy()
            got = codes[where, :, at]
            # the elements' values, so a zero may have either sign: of a head that holds an
            # infinity the others are products with 0, whose sign goes by their order
            assert np.array_equal(mx_ref.values(mx_ref.unpack(got) if fmt == "fp4" else got, sc, fmt), mx_ref.values(c, sc, fmt),
                                  equal_nan=True)
            assert np.array_equal(scales[where, :, :, at], sc)
            # the other places are as they were
            codes[where, :, at], scales[where, :, :, at] = 77, 77
            assert (codes == 77).all() and (scales == 77).all()
        before = Q.clone()
        again = cache.append(Q, K, V, _dev(positions), _dev(slots.astype(np.int64)), _dev(freqs), *on, eps=1e-5,
                             interleaved=interleaved, out=Q)
        assert again is Q and torch.equal(Q, q) and (n == 1 or (rot == 0 and not normed) or not torch.equal(Q, before))


def test_append_rounds_once():
    """A key just beside the border of two elements goes to its own side: in fp32
    it would lie on the border, and fall to the even element."""
    import torch
    from paper_2002_09049_amd import mpq
    cache = mpq.MXCache.empty(1, 16, 1, 32, "fp8")
    # 1.0625 lies half way from 1 to 1.125; 1.1875 from 1.125 to 1.25.  Weights in
    # fp32 times keys in fp32: 1.0625 + 2^-26, and 1.1875 - 2^-26 or so, in fp64.
    x = np.zeros((1, 1, 32), np.float32)
    x[0, 0, :3] = 448.0, 1 + 2.0 ** -13, 1 - 2.0 ** -13
    w = np.ones(32, np.float32)
    w[1] = np.float32(1.0625) * np.float32(1 - 2.0 ** -13 + 2.0 ** -23)
    w[2] = np.float32(1.1875) * np.float32(1 + 2.0 ** -13)
    exact = x[0, 0].astype(np.float64) * w / np.sqrt((x[0, 0].astype(np.float64) ** 2).mean() + 1e-6)
    t = [_dev(x) for _ in "qkv"]
    cache.append(*t, _dev(np.zeros(1, np.int32)), _dev(np.zeros(1, np.int64)), _dev(np.zeros(0)), _dev(w), _dev(w))
    c, s = mx_ref.quantize(exact[None, None], "fp8")
    assert np.array_equal(cache.tensors[0][0, :, 0].cpu().numpy(), c[0]) and cache.tensors[2][0, 0, 0, 0].item() == s[0, 0, 0]
    torch.cuda.synchronize()


def _keys_beside_borders(fmt, dtype, dim, rot, normed, interleaved):
    """(keys [1, 1, dim], positions, freqs, weight) whose turned values, in 64 bits,
    lie beside borders between two elements, nearer than fp32 can tell, on the side
    away from the even one; in both directions, of either sign."""
    vals = mx_ref.elements(fmt)
    lo = np.arange(len(vals) // 2, len(vals) - 1)   # of the upper half, where a block's scale is 1
    border = (vals[lo] + vals[lo + 1]) / 2
    rng = np.random.default_rng(dim + rot)
    x = np.zeros((1, 1, dim))
    if normed:
        x[0, 0] = _f64(_dev(rng.uniform(0.5, 2.0, dim), _dt(dtype)))
        root = np.sqrt((x[0, 0] ** 2).mean() + float(np.float32(1e-6)))
        w = np.ones(dim, np.float32)
        for i in range(dim):
            if i % 32 == 0:
                w[i] = vals[-1] * root / x[0, 0, i]   # the block's largest
                continue
            near = (border * root / x[0, 0, i]).astype(np.float32)
            off = near.astype(np.float64) * x[0, 0, i] / root / border - 1
            good = np.flatnonzero((np.abs(off) > 1e-11) & (np.abs(off) < 2.0 ** -26) & ((off > 0) == (lo % 2 == 0)))
            if len(good):
                w[i] = near[good[i % len(good)]] * rng.choice((-1, 1))
        return x, np.zeros(1, np.int32), np.zeros(0), w
    # cos 2^-14 is 1 - 2^-29, sin 2^-14 about 2^-14: a border b with a partner of 0 turns to
    # b - 2^-29 b, with one of -2^-13 b to b + 2^-27 b - 2^-29 b
    half = rot // 2
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, half), slice(half, rot))
    take = rng.permutation(np.arange(half) % len(lo))
    a = border[take] * rng.choice((-1, 1), half)
    b = np.where(lo[take] % 2 == 0, -a * 2.0 ** -13, 0.0)
    a[::8], b[::8] = vals[-1], 0.0   # the blocks' largest
    x[0, 0, first], x[0, 0, second] = a, b
    return x, np.ones(1, np.int32), np.full(half, 2.0 ** -14), None


@pytest.mark.parametrize("n", [1, 4096])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("dim,rot,normed,interleaved", [(64, 64, False, False), (64, 32, False, False), (96, 64, False, True),
                                                        (256, 256, False, False), (32, 0, True, False), (128, 0, True, False),
                                                        (80, 0, True, False)])
def test_append_rounds_keys_to_their_elements_alone(dim, rot, normed, interleaved, fmt, dtype, n):
    """A key just beside the border of two elements goes to its own side; by way of
    fp32 it would lie on the border, and fall to the even element."""
    import torch
    from paper_2002_09049_amd import mpq
    x, positions, freqs, w = _keys_beside_borders(fmt, dtype, dim, rot, normed, interleaved)
    exact, _ = ref.turned(x, positions, freqs, w, float(np.float32(1e-6)), interleaved)
    c, s = mx_ref.quantize(mx_ref.padded(exact, 32), fmt)
    short, _ = mx_ref.quantize(mx_ref.padded(exact.astype(np.float32).astype(np.float64), 32), fmt)
    # what a rounding in between would change: both up and down
    top = 7 if fmt == "fp4" else 127
    step = (short & top).astype(int) - (c & top)
    assert (step > 0).sum() >= 2 and (step < 0).sum() >= 2 and np.abs(step).max() == 1
    assert np.array_equal(_f64(_dev(x, _dt(dtype))), x)
    cache = mpq.MXCache.empty(n // 16 + 1, 16, 1, dim, fmt)
    t = [_dev(np.repeat(x, n, 0), _dt(dtype)) for _ in "qkv"]
    on = None if w is None else _dev(w)
    cache.append(*t, _dev(np.repeat(positions, n)), _dev(np.arange(n)), _dev(freqs), on, on, interleaved=interleaved)
    codes, scales = cache.tensors[0].cpu().numpy(), cache.tensors[2].cpu().numpy()
    at = np.arange(n)
    got = codes[at // 16, 0, at % 16]
    got = mx_ref.unpack(got) if fmt == "fp4" else got
    zero = (c[0, 0] & top) == 0   # of either sign
    assert (np.where(zero, got & top, got) == np.where(zero, 0, c[0, 0])).all()
    assert (scales[at // 16, 0, :, at % 16] == s[0, 0]).all()


def test_rotate_past_32_bit_offsets():
    """Tokens 2^31 elements apart."""
    import torch
    from paper_2002_09049_amd import mpq
    rng = np.random.default_rng(0)
    far = 2 ** 31 + 64
    wide = torch.zeros((far + 256,), dtype=torch.bfloat16, device="cuda")
    Q = torch.as_strided(wide, (2, 2, 64), (far, 64, 1))
    x = _heads(rng, 2, 2, 64, "bf16", 0)
    Q.copy_(x)
    p, f = _dev(np.array([5, 1000], np.int32)), _dev(_freqs(64))
    q, k = mpq.mx_rotate(Q, Q, p, f)
    want, _ = mpq.mx_rotate(x, x, p, f)
    assert torch.equal(q, want) and torch.equal(k, want)
    to = torch.as_strided(wide, (2, 1, 64), (far, 64, 1), 128)
    mpq.mx_rotate(x, x[:, :1].contiguous(), p, f, out=(q, to))
    assert torch.equal(to, want[:, :1]) and torch.equal(Q, x)
    del wide, Q, to
    torch.cuda.empty_cache()


def test_rotate_past_one_launch_dimension():
    """More workgroups than go in one row of a grid: 2^22 tokens and some."""
    import torch
    from paper_2002_09049_amd import mpq
    torch.manual_seed(0)
    n = 2 ** 22 + 9
    x = torch.randn((n, 2, 8), device="cuda").bfloat16()
    p = torch.arange(n, device="cuda", dtype=torch.int32)
    f = _dev(_freqs(8))
    q, k = mpq.mx_rotate(x[:, :1], x[:, 1:], p, f)
    for part in (slice(0, 100), slice(2 ** 22 - 50, n)):
        want = mpq.mx_rotate(x[part, :1], x[part, 1:], p[part].contiguous(), f)
        assert torch.equal(q[part], want[0]) and torch.equal(k[part], want[1])


def test_rotate_and_append_many_tokens():
    """More tokens and heads than one row of anything; against torch in 64 bits."""
    import torch
    from paper_2002_09049_amd import mpq
    torch.manual_seed(0)
    n, heads, kv, dim = 20011, 12, 3, 96
    Q, K = (torch.randn((n, h, dim), device="cuda").half() for h in (heads, kv))
    positions = torch.randint(0, 100000, (n,), device="cuda", dtype=torch.int32)
    freqs = _dev(_freqs(dim))
    got = mpq.mx_rotate(Q, K, positions, freqs)
    angle = (positions.double()[:, None] * freqs)[:, None]
    for g, x in zip(got, (Q, K)):
        a, b = x.double().chunk(2, -1)
        y = torch.cat((a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()), -1)
        bound = 20 * E * (a.abs() + b.abs()).repeat(1, 1, 2) + HALF["f16"] * y.abs() + TINY["f16"]
        assert ((g.double() - y).abs() <= bound).all()


# ---------------------------------------------------------------- route


def _check_route(x, k, renorm, dtype, got):
    """x: the logits' values as the call reads them, fp64."""
    n, experts = x.shape
    want = ref.route(x, k, renorm)
    got = [t.cpu().numpy() for t in got]
    for g, w, name in zip(got, want, ("chosen", "", "order", "place", "offsets")):
        if name:
            assert np.array_equal(g, w), name
    if n == 0:
        return
    v = np.where(np.isfinite(x), x, np.nan)
    with np.errstate(all="ignore"):
        spread = np.nan_to_num(np.nanmax(v, 1) - np.nanmin(np.where(v > np.nanmax(v, 1, keepdims=True) - 110, v, np.nan), 1))
    limit = E * (2 * spread + 2 * (experts / 64 + 6) + 8)[:, None] * want[1] + 2.0 ** -126
    assert (np.abs(got[1] - want[1]) <= limit).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,experts,k", [(1, 1, 1), (1, 8, 2), (4, 64, 8), (63, 60, 4), (64, 65, 6), (65, 128, 8), (130, 129, 1),
                                         (1000, 256, 8), (300, 257, 12), (777, 512, 64), (200, 1000, 10), (129, 1024, 64),
                                         (5000, 5, 5), (70, 64, 64)])
def test_route(n, experts, k, dtype):
    from paper_2002_09049_amd import mpq
    rng = np.random.default_rng(n + experts)
    x = rng.standard_normal((n, experts)) * 3 + rng.standard_normal(experts)
    wide = _dev(np.concatenate([np.full((n, 3), 1e4), x, np.full((n, 2), 1e4)], 1), _dt(dtype))
    logits = wide[:, 3:3 + experts]
    for renorm in (True, False):
        _check_route(_f64(logits), k, renorm, dtype, mpq.mx_route(logits, k, renorm))


@pytest.mark.parametrize("n", [3, 200])
def test_route_ties_and_values_that_are_not_finite(n):
    from paper_2002_09049_amd import mpq
    rng = np.random.default_rng(n)
    x = rng.integers(-2, 3, (n, 70)).astype(np.float64)
    x[x == 0] = np.where(rng.random((x == 0).sum()) < 0.5, 0.0, -0.0)
    x[0], x[1, ::2], x[2, 5] = -np.inf, np.nan, np.inf
    if n > 3:
        x[3], x[4, :], x[5, 10:30] = np.nan, 7.0, np.inf
        x[6, :] = np.where(np.arange(70) % 3 == 0, 3e38, -3e38)
    for dtype in ("f32", "bf16"):
        logits = _dev(x, _dt(dtype))
        for renorm in (True, False):
            _check_route(_f64(logits), 9, renorm, dtype, mpq.mx_route(logits, 9, renorm))


def test_route_all_to_one_expert_and_none():
    """One expert takes all; no tokens at all."""
    import torch
    from paper_2002_09049_amd import mpq
    x = np.zeros((5000, 33))
    x[:, 17] = 1.0
    _check_route(x, 2, True, "f32", mpq.mx_route(_dev(x, torch.float32), 2))
    chosen, weights, order, place, offsets = mpq.mx_route(torch.zeros((0, 33), device="cuda"), 2)
    assert offsets.tolist() == [0] * 34 and chosen.shape == (0, 2) and order.numel() == 0


def test_route_many_tokens():
    """As many as a call takes."""
    import torch
    from paper_2002_09049_amd import mpq
    torch.manual_seed(1)
    n, experts, k = 2 ** 20, 8, 2
    logits = torch.randn((n, experts), device="cuda")
    chosen, weights, order, place, offsets = mpq.mx_route(logits, k)
    want = torch.sort(logits, dim=-1, descending=True, stable=True)[1][:, :k]
    assert torch.equal(chosen.long(), want)
    flat = want.reshape(-1)
    assert torch.equal(order.long(), torch.argsort(flat, stable=True))
    assert torch.equal(order.long()[place.reshape(-1).long()], torch.arange(n * k, device="cuda"))
    assert offsets.tolist() == [0] + torch.cumsum(torch.bincount(flat, minlength=experts), 0).tolist()


def _check_long_route(x, k, renorm, got):
    """x: the logits' values, fp64.  Weights, in units of 2^-24: a logit's difference
    from the top and expf (2 steps) in numerator and denominator, 2 spread + 8; a
    lane's sum of up to 16 parts and 6 steps between lanes, 22; the quotient, 1."""
    chosen, w, order, place, offsets = ref.route(x, k, renorm)
    got = [t.cpu().numpy() for t in got]
    for g, want, name in zip(got, (chosen, None, order, place, offsets), ("chosen", "", "order", "place", "offsets")):
        if name:
            assert np.array_equal(g, want), (name, np.argwhere(g != want)[:5].tolist())
    top = np.where(np.isnan(x), -np.inf, x).max(1, keepdims=True)
    with np.errstate(invalid="ignore"):
        below = top - x
    spread = np.where(np.isfinite(below) & (below < 110), below, 0.0).max(1, keepdims=True)
    bad = ~(np.abs(got[1] - w) <= E * (2 * spread + 31) * w + 2.0 ** -126)
    assert not bad.any(), (np.argwhere(bad)[:5].tolist(), got[1][bad][:5], w[bad][:5])


# 64 tokens a workgroup, the last one of one, or of all but one; experts at and beside
# every width of a lane's keys; choices that several tokens a wavefront can hold and not
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k", [1, 8, 16, 17])
@pytest.mark.parametrize("n,experts", [(4097, 16), (4159, 17), (4097, 64), (4160, 65), (4159, 100), (4097, 128), (4161, 129),
                                       (4159, 256), (4097, 257), (4161, 511), (4097, 512), (4159, 513), (4097, 1000), (4161, 1024)])
def test_route_long(n, experts, k, dtype):
    from paper_2002_09049_amd import mpq
    if k > experts:
        k = experts
    rng = np.random.default_rng(n + experts + k)
    x = rng.standard_normal((n, experts)) * 3 + rng.standard_normal(experts)
    # ties of whole rows' parts, zeros of both signs, and values that are not finite
    x[5::7] = np.round(x[5::7])
    x[1, :], x[2, ::2], x[3, experts // 2], x[n - 1, :] = -np.inf, np.nan, np.inf, 7.0
    x[4, experts // 3:], x[6, :], x[7, ::3] = np.inf, np.nan, -np.inf
    x[8, :] = np.where(np.arange(experts) % 2 == 0, 0.0, -0.0)
    wide = np.concatenate([np.full((n, 1), 1e4), x, np.full((n, 2), 1e4)], 1)
    logits = _dev(wide, _dt(dtype))[:, 1:1 + experts]
    x = _f64(logits)
    for renorm in (True, False):
        _check_long_route(x, k, renorm, mpq.mx_route(logits, k, renorm))


@pytest.mark.parametrize("experts", [1, 2, 4, 5, 8, 33, 128])
@pytest.mark.parametrize("n", [65, 100, 496, 513, 4096, 4097, 8200, 65472])
def test_route_counts_of_few_and_many_workgroups(n, experts):
    """Fewer workgroups' counts than threads to add them, as many, and more, of few
    experts and many; and all tokens to one expert, whose sum takes 16 bits whole."""
    import torch
    from paper_2002_09049_amd import mpq
    x = torch.randn((n, experts), generator=torch.Generator("cuda").manual_seed(n + experts), device="cuda")
    crowd = torch.zeros_like(x)
    crowd[:, experts // 2] = 1.0
    for logits in (x, crowd):
        k = min(2, experts)
        chosen, _, order, place, offsets = mpq.mx_route(logits, k)
        want = torch.sort(logits, dim=-1, descending=True, stable=True)[1][:, :k]
        flat = want.reshape(-1)
        assert torch.equal(chosen.long(), want) and torch.equal(order.long(), torch.argsort(flat, stable=True))
        assert torch.equal(order.long()[place.reshape(-1).long()], torch.arange(n * k, device="cuda"))
        assert offsets.tolist() == [0] + torch.cumsum(torch.bincount(flat, minlength=experts), 0).tolist()


@pytest.mark.parametrize("n,experts,k,dtype", [(4096, 1000, 9, "f32"), (4095, 1024, 64, "bf16"), (70000, 50, 6, "f16"),
                                               (65473, 3, 2, "bf16"), (40000, 257, 8, "bf16"), (37777, 511, 10, "f32")])
def test_route_counts_summed_apart(n, experts, k, dtype):
    """So many tokens and experts that a launch of its own sums the counts."""
    from paper_2002_09049_amd import mpq
    rng = np.random.default_rng(n)
    logits = _dev(rng.standard_normal((n, experts)) * 2 + rng.standard_normal(experts), _dt(dtype))
    mpq.timing_enable(True)
    try:
        got = mpq.mx_route(logits, k)
        names = {name for name, _ in mpq.timing_read()}
    finally:
        mpq.timing_enable(False)
    assert "mx_sum_kernel" in names, names
    _check_long_route(_f64(logits), k, True, got)


# ---------------------------------------------------------------- experts


def _drawn(rng, shape):
    """As _activations, drawn on the device."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(int(rng.integers(2 ** 31)))
    x = torch.randn(shape, generator=g, device="cuda") * torch.exp(torch.randn(shape[-1:], generator=g, device="cuda"))
    return torch.where(torch.rand(shape, generator=g, device="cuda") < 0.02, torch.zeros_like(x), x)


def _weights(rng, experts, c, d):
    from paper_2002_09049_amd import mpq
    codes, scales = mpq.mx_quantize(_drawn(rng, (experts * c, d)) / d ** 0.5)
    return codes.reshape(experts, c, -1), scales.reshape(experts, c, -1)


def _expert_products(X, codes, scales, offsets, order, k, bias):
    """(Y, its bound less the output's rounding), and the rows of groups, on the
    device in 64 bits."""
    import torch
    from paper_2002_09049_amd import mpq
    n, d = X.shape
    x = mpq.mx_dequantize(*mpq.mx_quantize(X), d).double()
    x = torch.cat([x, torch.zeros((1, d), dtype=torch.float64, device="cuda")])
    m = n if order is None else order.numel()
    rows = torch.arange(m, device="cuda") if order is None else torch.where(order < 0, n, torch.clamp(order // k, max=n)).long()
    y = torch.zeros((m, codes.shape[1]), dtype=torch.float64, device="cuda")
    size, live = torch.zeros_like(y), torch.zeros((m,), dtype=torch.bool, device="cuda")
    for e, (a, b) in enumerate(ref.groups(offsets.cpu().numpy(), m)):
        if a < b:
            w = mpq.mx_dequantize(codes[e].contiguous(), scales[e].contiguous(), d).double()
            y[a:b], size[a:b] = x[rows[a:b]] @ w.t(), x[rows[a:b]].abs() @ w.abs().t()
            live[a:b] = True
            if bias is not None:
                y[a:b] += bias[e].double()
                size[a:b] += bias[e].double().abs()
    return y, (128 + -(-d // 128) + 16) * E * size, live


def _check_experts(rng, n, k, experts, c, d, dtype, out_dtype, counts=None, bias=False, gather=True, layout=0, tail=0):
    import torch
    from paper_2002_09049_amd import mpq
    m = n * k if gather else n
    codes, scales = _weights(rng, experts, c, d)
    if counts is None:
        counts = rng.multinomial(m - tail, rng.dirichlet(np.full(experts, 0.7)))
    first = rng.integers(0, tail + 1)
    offsets = _dev(np.concatenate([[first], first + np.cumsum(counts)]).astype(np.int32))
    order = _dev(rng.permutation(m).astype(np.int32)) if gather else None
    X = torch.full((n, d + 3 * layout), 9.0, dtype=_dt(dtype), device="cuda")[:, layout:layout + d]
    X.copy_(_drawn(rng, (n, d)))
    b = _dev(rng.standard_normal((experts, c)).astype(np.float32)) if bias else None
    wide = torch.full((m + 2, c + 3 * layout), 3.5, dtype=_dt(out_dtype), device="cuda")
    Y = wide[1:1 + m, layout:layout + c]
    mpq.mx_experts(X, codes, scales, offsets, order=order, k=k if gather else 1, bias=b, out=Y)
    y, bound, live = _expert_products(X, codes, scales, offsets, order, k if gather else 1, b)
    bound = bound + HALF[out_dtype] * y.abs() + TINY[out_dtype]
    bad = ((Y.double() - y).abs() > bound) & live[:, None]
    assert not bad.any(), (bad.nonzero()[:5].tolist(), Y[bad][:5].tolist(), y[bad][:5].tolist())
    keep = wide.clone()
    keep[1:1 + m, layout:layout + c][live] = 3.5
    assert (keep == 3.5).all()
    # a workspace of the caller's, and new memory: the same bits
    space = torch.empty((mpq.mx_experts_workspace(n, m, experts, c, d),), dtype=torch.uint8, device="cuda")
    again = mpq.mx_experts(X, codes, scales, offsets, order=order, k=k if gather else 1, bias=b, workspace=space, dtype=_dt(out_dtype))
    assert torch.equal(again[live], Y[live])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,k,experts,c,d", [
    (1, 1, 1, 1, 1), (1, 8, 64, 33, 200), (2, 2, 5, 17, 31), (4, 6, 60, 130, 513), (4, 20, 30, 16, 96), (5, 3, 7, 100, 1000),
    (48, 6, 60, 64, 384), (33, 2, 3, 129, 127), (77, 3, 5, 200, 640), (300, 2, 9, 257, 129), (500, 4, 13, 70, 2047),
    (700, 2, 4, 300, 512), (1500, 2, 5, 65, 260), (64, 1, 1024, 20, 64), (9, 8, 1000, 5, 64)])
def test_experts(n, k, experts, c, d, dtype):
    rng = np.random.default_rng(n + c + d)
    out = {"f32": "bf16", "f16": "f32", "bf16": "f16"}[dtype]
    _check_experts(rng, n, k, experts, c, d, dtype, dtype)
    _check_experts(rng, n, k, experts, c, d, dtype, out, bias=True, layout=1, tail=min(3, n * k - 1))
    _check_experts(rng, n, 1, experts, c, d, dtype, dtype, bias=True, gather=False)


WAYS = [
    ("mx_experts_token_kernel", 1, 8, 16, 2500, 300), ("mx_experts_token_kernel", 4, 16, 40, 1100, 600),
    ("mx_experts_few_kernel", 60, 1, 50, 300, 700), ("mx_experts_few_kernel", 60, 1, 50, 1030, 3000),
    ("mx_experts_few_kernel", 100, 1, 9, 200, 8200), ("mx_experts_few_kernel", 4, 16, 64, 5001, 1000),
    ("mx_experts_tile_kernel<2,1>", 600, 1, 21, 2050, 260), ("mx_experts_tile_kernel<2,1>", 700, 4, 70, 130, 2100),
    ("mx_experts_tile_kernel<2,2>", 4000, 2, 40, 400, 1000), ("mx_experts_tile_kernel<2,2>", 3000, 1, 4, 700, 900),
    ("mx_experts_stay_kernel", 4100, 2, 2, 2050, 200), ("mx_experts_stay_kernel", 8000, 3, 7, 1100, 1290),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kernel,n,k,experts,c,d", WAYS)
def test_experts_by_every_kernel(kernel, n, k, experts, c, d, dtype):
    """Sizes at which the rule takes each kernel, several tiles a workgroup where
    those stay; all types of outputs, strided, with and without bias and order."""
    from paper_2002_09049_amd import mpq
    rng = np.random.default_rng(n + c + d)
    for out, bias, gather, layout, tail in ((dtype, False, True, 0, 0), ("f32", True, True, 1, 2), ("bf16", True, n > 4, 0, 0),
                                            ("f16", False, True, 1, 0)):
        mpq.timing_enable(True)
        try:
            _check_experts(rng, n, k, experts, c, d, dtype, out, bias=bias, gather=gather, layout=layout, tail=tail)
            names = {name for name, _ in mpq.timing_read()}
        finally:
            mpq.timing_enable(False)
        if gather:
            assert kernel in names, names


@pytest.mark.parametrize("counts", [[0, 0, 0, 0], [0, 64, 0, 0], [16, 17, 15, 16], [1, 0, 62, 1], [0, 0, 0, 64], [3, 0, 0, 2]])
def test_experts_without_rows(counts):
    rng = np.random.default_rng(sum(counts))
    for n in (16, 4):   # (4 tokens: inside one launch)
        _check_experts(rng, n, 64 // n, 4, 40, 300, "bf16", "bf16", counts=np.array(counts), tail=64 - sum(counts))


@pytest.mark.parametrize("rows", [15, 16, 17, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300])
def test_experts_at_the_pieces_edges(rows):
    """Groups one below, at, and one above a tile, whatever kernel the mean picks."""
    rng = np.random.default_rng(rows)
    counts = np.array([rows, 1, 0, rows - 1, rows + 1])
    _check_experts(rng, int(counts.sum()), 1, 5, 200, 520, "bf16", "f32", counts=counts)
    _check_experts(rng, int(counts.sum()), 1, 5, 260, 140, "f16", "f16", counts=counts, gather=False)


@pytest.mark.parametrize("n", [3, 40, 500])
def test_experts_offsets_and_orders_that_name_nothing(n):
    """Offsets that fall or leave [0, m], and choices of no row."""
    import torch
    from paper_2002_09049_amd import mpq
    rng = np.random.default_rng(n)
    codes, scales = _weights(rng, 6, 40, 200)
    X = _dev(_activations(rng, (n, 200)), torch.bfloat16)
    m = 2 * n
    order = rng.permutation(m).astype(np.int32)
    order[0], order[m // 2], order[m - 1] = -1, 2 ** 31 - 1, 2 * n
    order = _dev(order)
    for offsets in ([-4, 2, 1, m // 2, m // 3, m - 1, m + 9], [1, 1, 3, 2, 5, 4, 2], [m, 0, 0, 0, 0, 0, m], [0] * 7,
                    [-9, -8, -7, -6, -5, -4, -3], [m + 1] * 7, [0, 2 ** 31 - 1, 0, 0, 0, 0, 0]):
        off = _dev(np.array(offsets, np.int32))
        out = torch.full((m, 40), 3.5, device="cuda")
        mpq.mx_experts(X, codes, scales, off, order=order, k=2, out=out)
        y, bound, live = _expert_products(X, codes, scales, off, order, 2, None)
        assert ((out.double() - y).abs() <= bound + HALF["f32"] * y.abs() + TINY["f32"])[live].all(), offsets
        assert (out[~live] == 3.5).all(), offsets


def test_experts_rows_that_are_not_finite():
    """A row with an infinity or a NaN has NaN in its products and in no others."""
    import torch
    from paper_2002_09049_amd import mpq
    for n in (3, 30, 300):
        rng = np.random.default_rng(n)
        codes, scales = _weights(rng, 4, 70, 130)
        X = _dev(_activations(rng, (n, 130)), torch.float32)
        off = _dev(np.array([0, n // 3, n // 3, 2 * n // 3, n], np.int32))
        clean = mpq.mx_experts(X, codes, scales, off)
        X[1, 7], X[n - 1, 129] = float("inf"), float("nan")
        y = mpq.mx_experts(X, codes, scales, off)
        assert y[1].isnan().all() and y[n - 1].isnan().all()
        y[1], y[n - 1] = clean[1], clean[n - 1]
        assert torch.equal(y, clean)


def test_experts_past_32_bit_offsets():
    """Y and the weights' codes of more than 2^31 elements and bytes."""
    import torch
    from paper_2002_09049_amd import mpq
    rng = np.random.default_rng(3)
    n, c, d = 5000, 128, 256
    codes, scales = _weights(rng, 3, c, d)
    X = _dev(_activations(rng, (n, d)), torch.bfloat16)
    off = _dev(np.array([0, 1500, 4000, n], np.int32))
    want = mpq.mx_experts(X, codes, scales, off)
    ld = 2 ** 31 // n + 512
    wide = torch.empty((n, ld), dtype=torch.bfloat16, device="cuda")
    mpq.mx_experts(X, codes, scales, off, out=wide[:, :c])
    assert torch.equal(wide[:, :c], want)
    del wide
    # experts' codes beyond 2^31 bytes: 1000 experts of 2.6 MB
    E_, C_, D_ = 1000, 1300, 4096
    big = torch.zeros((E_, C_, D_ // 2), dtype=torch.uint8, device="cuda")
    bs = torch.full((E_, C_, D_ // 32), 127, dtype=torch.uint8, device="cuda")
    assert big.numel() > 2 ** 31
    held = _weights(rng, 1, C_, D_)
    big[E_ - 1], bs[E_ - 1] = held[0][0], held[1][0]
    for n in (2, 40, 700):
        X = _dev(_activations(rng, (n, D_)), torch.bfloat16)
        off = torch.zeros((E_ + 1,), dtype=torch.int32, device="cuda")
        off[E_] = n
        y, bound, _ = _expert_products(X, *held, torch.tensor([0, n], device="cuda"), None, 1, None)
        got = mpq.mx_experts(X, big, bs, off)
        assert ((got.double() - y).abs() <= bound + HALF["bf16"] * y.abs() + TINY["bf16"]).all()
    torch.cuda.empty_cache()


# ---------------------------------------------------------------- combine


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,k,c", [(1, 1, 1), (1, 8, 2048), (61, 3, 999), (7, 2, 8), (300, 10, 17), (5, 64, 130), (3, 0, 40), (2000, 4, 256)])
def test_combine(n, k, c, dtype):
    import torch
    from paper_2002_09049_amd import mpq
    rng = np.random.default_rng(n + k + c)
    m = n * k + 3
    wide = _dev(_activations(rng, (m, c + 5)), _dt(dtype))
    Y = wide[:, 3:3 + c]
    place = rng.permutation(m)[:n * k].reshape(n, k)
    weights = rng.random((n, k)).astype(np.float32)
    if n > 3 and k > 1:
        place[1, 0], place[2, 1], place[3] = -1, m, place[3, 0]
        weights[1, 0] = np.nan   # of a place that takes no part
    R = _dev(_activations(rng, (n, c)), _dt(dtype))
    rows = np.concatenate([_f64(Y), np.zeros((1, c))])[np.where((place < 0) | (place >= m), m, place)]
    with np.errstate(invalid="ignore"):
        terms = rows * np.where((place < 0) | (place >= m), 0.0, weights.astype(np.float64))[..., None]
    for residual in (None, R):
        for out_dtype in (dtype, "f32"):
            got = mpq.mx_combine(Y, _dev(place.astype(np.int32)), _dev(weights), residual, dtype=_dt(out_dtype))
            r = np.zeros((n, c)) if residual is None else _f64(R)
            _near(got, r + terms.sum(1), (k + 1) * E * (np.abs(r) + np.abs(terms).sum(1)), out_dtype)
    want = mpq.mx_combine(Y, _dev(place.astype(np.int32)), _dev(weights), R)
    got = mpq.mx_combine(Y, _dev(place.astype(np.int32)), _dev(weights), R, out=R)
    assert got is R and torch.equal(R, want)


def test_combine_past_32_bit_offsets():
    import torch
    from paper_2002_09049_amd import mpq
    c = 4096
    m = 2 ** 31 // c + 40
    Y = torch.zeros((m, c), dtype=torch.bfloat16, device="cuda")
    Y[m - 7:] = torch.randn((7, c), device="cuda").bfloat16()
    place = _dev(np.array([[m - 1, m - 5], [m - 3, 0]], np.int32))
    w = _dev(np.array([[0.5, 2.0], [1.0, 1.0]], np.float32))
    got = mpq.mx_combine(Y, place, w, dtype=torch.float32)
    assert torch.equal(got[0], 0.5 * Y[m - 1].float() + 2.0 * Y[m - 5].float()) and torch.equal(got[1], Y[m - 3].float())
    del Y
    torch.cuda.empty_cache()


# ---------------------------------------------------------------- together


class _Step:
    """One decoding step of a layer: plan, append, attend, route, experts, combine."""

    def __init__(self, batch, fmt="fp8", seed=0):
        import torch
        from paper_2002_09049_amd import mpq
        self.mpq, self.torch, self.batch = mpq, torch, batch
        rng = np.random.default_rng(seed)
        self.heads, self.kv, self.dim, self.page, self.columns, self.experts, self.k = 8, 2, 64, 16, 6, 12, 3
        self.width = self.heads * self.dim
        self.cache = mpq.MXCache.empty(batch * self.columns, self.page, self.kv, self.dim, fmt)
        self.up = _weights(rng, self.experts, 2 * 320, self.width)
        self.down = _weights(rng, self.experts, self.width, 320)
        self.router = _dev(rng.standard_normal((self.width, self.experts)) / np.sqrt(self.width), torch.bfloat16)
        self.weight = _dev(rng.uniform(0.5, 1.5, self.dim).astype(np.float32))
        self.freqs = _dev(_freqs(self.dim))
        self.free = _dev(rng.permutation(batch * self.columns).astype(np.int32))
        self.table = torch.full((batch, self.columns), -1, dtype=torch.int32, device="cuda")
        self.cached = _dev(np.zeros(batch, np.int32))
        self.fresh = _dev(np.ones(batch, np.int32))
        self.taken = _dev(np.zeros(1, np.int32))

    def __call__(self, qkv, x):
        mpq, torch = self.mpq, self.torch
        q, k, v = qkv.split([self.heads, self.kv, self.kv], 1)
        slots, positions, starts, lengths, taken = mpq.mx_plan(self.cached, self.fresh, self.table, self.free, self.taken,
                                                               self.page, self.batch)
        q = self.cache.append(q, k, v, positions, slots, self.freqs, self.weight, self.weight)
        x = x + self.cache.attend(q, self.table, lengths).reshape(self.batch, -1)
        _, weights, order, place, offsets = mpq.mx_route(x @ self.router, self.k)
        gate, up = mpq.mx_experts(x, *self.up, offsets, order, self.k).chunk(2, -1)
        y = mpq.mx_experts((torch.nn.functional.silu(gate.float()) * up.float()).bfloat16(), *self.down, offsets)
        y = mpq.mx_combine(y, place, weights, x)
        self.cached.copy_(lengths)
        self.taken.copy_(taken)
        return y


@pytest.mark.parametrize("batch", [1, 5, 70])
def test_steps_together_in_a_graph(batch):
    """Steps one after the other, eager and as replays of a captured one (side by
    side, with their own state): the same bits, and the plan that the steps give."""
    import torch
    eager, captured = _Step(batch), _Step(batch)
    g = torch.Generator(device="cuda").manual_seed(batch)
    inputs = [(torch.randn((batch, 12, 64), generator=g, device="cuda").bfloat16(),
               torch.randn((batch, 512), generator=g, device="cuda").bfloat16()) for _ in range(20)]
    qkv, x = (t.clone() for t in inputs[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = captured(qkv, x)   # warm up: the first step
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(want, eager(*inputs[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = captured(qkv, x)
    for i, (a, b) in enumerate(inputs[1:], 1):
        qkv.copy_(a)
        x.copy_(b)
        graph.replay()
        want = eager(a, b)
        assert torch.equal(y, want), i
        assert torch.equal(captured.table, eager.table) and captured.cached.tolist() == [i + 1] * batch
        assert y.isfinite().all()
    used = eager.table[:, :2].cpu().numpy()   # 20 tokens: two pages each, all distinct
    assert (eager.table[:, 2:] == -1).all() and len(np.unique(used)) == 2 * batch
    assert eager.taken.tolist() == [2 * batch]
    say(f"{batch} sequences: steps and replays agree")


def test_calls_on_another_stream():
    """With stream=, work and memory are the stream's: the same bits as on the
    current one, which is busy."""
    import torch
    from paper_2002_09049_amd import mpq
    rng = np.random.default_rng(8)
    n, k, experts, c, d = 150, 2, 8, 96, 256
    codes, scales = _weights(rng, experts, c, d)
    X = _dev(_activations(rng, (n, d)), torch.bfloat16)
    logits = _dev(rng.standard_normal((n, experts)), torch.float32)
    Q, K = _heads(rng, n, 4, 64, "bf16", 0), _heads(rng, n, 2, 64, "bf16", 0)
    p, f = _dev(np.arange(n, dtype=np.int32)), _dev(_freqs(64))
    ints = [_dev(np.full(3, v, np.int32)) for v in (5, 50)]
    table = torch.full((3, 8), -1, dtype=torch.int32, device="cuda")
    free, taken = _dev(np.arange(64, dtype=np.int32)), _dev(np.zeros(1, np.int32))

    def calls(stream):
        plan = mpq.mx_plan(*ints, table, free, taken, 16, n, stream=stream)
        cache = mpq.MXCache.empty(n // 16 + 1, 16, 2, 64)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        q = cache.append(Q, K, K, p, p.long(), f, stream=stream)
        turned = mpq.mx_rotate(Q, K, p, f, stream=stream)
        route = mpq.mx_route(logits, k, stream=stream)
        y = mpq.mx_experts(X, codes, scales, route[4], route[2], k, stream=stream)
        z = mpq.mx_combine(y, route[3], route[1], stream=stream)
        return [*plan, table.clone() if stream is None else table, q, *turned, *route, y, z, *cache.tensors]

    want = calls(None)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    busy = torch.randn((4096, 4096), device="cuda")
    for _ in range(10):
        busy = busy @ busy * 1e-3
    got = calls(stream)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_every_call_on_another_stream():
    """With stream=, work and memory are the stream's: the same bits as on the
    current one, which is busy.  All inputs are there before either pass, and each
    pass has a page table, a cache and outputs of its own."""
    import torch
    from paper_2002_09049_amd import mpq
    rng = np.random.default_rng(9)
    n, k, experts, c, d = 150, 2, 8, 96, 256
    codes, scales = _weights(rng, experts, c, d)
    X = _dev(_activations(rng, (n, d)), torch.bfloat16)
    logits = _dev(rng.standard_normal((n, experts)), torch.float32)
    Q, K, V = (_heads(rng, n, h, 64, "bf16", 0) for h in (4, 2, 2))
    f = _dev(_freqs(64))
    cached, fresh = _dev(np.array([5, 40, 0], np.int32)), _dev(np.array([50, 1, 99], np.int32))
    held = np.full((3, 8), -1, np.int32)
    held[0, 0], held[1, :3] = 60, (61, 62, 63)
    free, taken = _dev(rng.permutation(60).astype(np.int32)), _dev(np.zeros(1, np.int32))
    tables = [_dev(held) for _ in range(2)]
    caches = [mpq.MXCache.empty(64, 16, 2, 64) for _ in range(2)]
    for cache in caches:
        for t in cache.tensors:
            t.fill_(77)
    stream = torch.cuda.Stream()
    busy = torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()

    def calls(table, cache, stream):
        plan = mpq.mx_plan(cached, fresh, table, free, taken, 16, n, stream=stream)
        slots, positions = plan[:2]
        q = cache.append(Q, K, V, positions, slots, f, stream=stream)
        turned = mpq.mx_rotate(Q, K, positions, f, stream=stream)
        route = mpq.mx_route(logits, k, stream=stream)
        y = mpq.mx_experts(X, codes, scales, route[4], route[2], k, stream=stream)
        z = mpq.mx_combine(y, route[3], route[1], stream=stream)
        return [*plan, table, q, *turned, *route, y, z, *cache.tensors]

    for _ in range(10):
        busy = busy @ busy * 1e-3
    got = calls(tables[0], caches[0], stream)
    with torch.cuda.stream(stream):   # (waits for this stream alone: the other is still busy)
        there = [t.cpu() for t in got]
    torch.cuda.synchronize()
    want = calls(tables[1], caches[1], None)
    torch.cuda.synchronize()
    assert len(got) == len(want)
    for i, (a, b, early) in enumerate(zip(want, got, there)):
        assert torch.equal(a, b) and torch.equal(a.cpu(), early), i
    slots, positions, starts, lengths, after, table = ref.plan(cached.tolist(), fresh.tolist(), held, free.tolist(), 0, 16, n)
    for a, b in zip(got, (slots, positions, starts, lengths, [after], table)):
        assert np.array_equal(a.cpu().numpy(), b)


def test_one_workspace_for_steps_of_every_size():
    """Allocated once, for the longest step: the shorter ones give what they give
    with new memory."""
    import torch
    from paper_2002_09049_amd import mpq
    rng = np.random.default_rng(10)
    experts, k, c, d = 1000, 3, 24, 130
    codes, scales = _weights(rng, experts, c, d)
    most = 4200
    X = _dev(_activations(rng, (most, d)), torch.bfloat16)
    logits = _dev(rng.standard_normal((most, experts)), torch.float32)
    routing = torch.empty((mpq.mx_route_workspace(most, experts, k),), dtype=torch.uint8, device="cuda")
    products = torch.empty((mpq.mx_experts_workspace(most, most * k, experts, c, d),), dtype=torch.uint8, device="cuda")
    for n in (most, 4097, 4096, 4095, 700, 341, 65, 64, 5, 4, 1):
        routing.fill_(n % 251)
        products.fill_(n % 251)
        got, want = mpq.mx_route(logits[:n], k, workspace=routing), mpq.mx_route(logits[:n], k)
        for a, b in zip(got, want):
            assert torch.equal(a, b), n
        y = mpq.mx_experts(X[:n], codes, scales, got[4], got[2], k, workspace=products)
        assert torch.equal(y, mpq.mx_experts(X[:n], codes, scales, got[4], got[2], k)), n


def test_refusals_of_the_binding():
    """Shapes, types and devices, before the library is called."""
    import torch
    from paper_2002_09049_amd import mpq
    i = torch.zeros(2, dtype=torch.int32, device="cuda")
    t = torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    x = torch.zeros((2, 3, 40), device="cuda")
    f = torch.zeros(20, dtype=torch.float64, device="cuda")
    codes = torch.zeros((3, 5, 64), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((3, 5, 4), dtype=torch.uint8, device="cuda")
    off, place, w = torch.zeros(4, dtype=torch.int32, device="cuda"), t[:, :2].contiguous(), torch.zeros((2, 2), device="cuda")
    y = torch.zeros((4, 5), device="cuda")
    cache = mpq.MXCache.empty(2, 16, 3, 40)
    bad = [
        lambda: mpq.mx_plan(i, i[:1], t, i, i[:1], 16, 4), lambda: mpq.mx_plan(i, i, t[:1], i, i[:1], 16, 4),
        lambda: mpq.mx_plan(i, i, t.long(), i, i[:1], 16, 4), lambda: mpq.mx_plan(i, i, t, i, i, 16, 4),
        lambda: mpq.mx_plan(i.long(), i, t, i, i[:1], 16, 4), lambda: mpq.mx_plan(i, i, t.t().contiguous().t(), i, i[:1], 16, 4),
        lambda: mpq.mx_plan(i, i.cpu(), t, i, i[:1], 16, 4),
        lambda: mpq.mx_rotate(x, x, i[:1], f), lambda: mpq.mx_rotate(x, x, i, f.float()), lambda: mpq.mx_rotate(x, x.half(), i, f),
        lambda: mpq.mx_rotate(x, x, i, f, q_weight=f[:20].float()), lambda: mpq.mx_rotate(x, x[..., :20], i, f),
        lambda: mpq.mx_rotate(x, x, i, f, out=(x, x.half())), lambda: mpq.mx_rotate(x.double(), x.double(), i, f),
        lambda: mpq.mx_rotate(x, x, i.cpu(), f),
        lambda: cache.append(x, x, x, i, i, f), lambda: cache.append(x, x, x[:, :2], i, i.long(), f),
        lambda: cache.append(x, x.half(), x, i, i.long(), f), lambda: cache.append(x, x, x, i, i.long()[:1], f),
        lambda: mpq.mx_route(y.double(), 2), lambda: mpq.mx_route(y[0], 2), lambda: mpq.mx_route(y, 2, out=(off,) * 5),
        lambda: mpq.mx_experts(y[:, :4], codes, scales, off[:3]), lambda: mpq.mx_experts(y, codes[..., :32], scales, off),
        lambda: mpq.mx_experts(y, codes, scales, off.long()), lambda: mpq.mx_experts(y, codes, scales, off, bias=w),
        lambda: mpq.mx_experts(y, codes, scales, off, order=t), lambda: mpq.mx_experts(y, codes, scales, off.cpu()),
        lambda: mpq.mx_combine(y, place, w[:1]), lambda: mpq.mx_combine(y, place.long(), w),
        lambda: mpq.mx_combine(y, place, w, residual=y), lambda: mpq.mx_combine(y, place, w, residual=y[:2].half()),
        lambda: mpq.mx_combine(y, place.cpu(), w)]
    for n, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {n} was taken")
    with pytest.raises(mpq.MPQError):
        mpq.mx_route(y, 6)
    with pytest.raises(mpq.MPQError):
        mpq.mx_plan(i, i, t, i, i[:1], 24, 4)
    with pytest.raises(mpq.MPQError):
        mpq.mx_rotate(x, x, i, f, x[0, 0], x[0, 0], eps=0.0)
