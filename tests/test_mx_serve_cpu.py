"""A serving step's calls without a GPU: what they refuse, before any HIP call,
the sizes they report, and the offsets and rings of the products by expert."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

import mx_serve_ref as ref
import test_mx_ring_cpu as ring

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2002_09049_amd", "csrc")


@pytest.fixture(scope="module")
def mpq():
    from paper_2002_09049_amd import mpq
    if not os.path.exists(mpq.LIB_PATH):
        from paper_2002_09049_amd import build
        build.build()
    mpq.load()
    return mpq


def _refused(mpq, fn, ok, changes):
    """Every change of one argument of a valid call is refused with a text."""
    for kw in changes:
        a = dict(ok)
        a.update(kw)
        assert set(kw) <= set(ok), kw
        assert fn(*a.values()) == mpq.MPQ_ERR_INVALID_ARG, kw
        assert mpq.last_error(), kw


def test_plan_refusals(mpq):
    ok = dict(cached=64, fresh=128, batch=2, table=256, table_ld=4, columns=4, free=512, n_free=8, taken=1024, page=16,
              tokens=9, slots=2048, positions=4096, starts=8192, lengths=16384, taken_out=32768, stream=None)
    bad = [dict(cached=None), dict(cached=66), dict(fresh=None), dict(fresh=66), dict(batch=-1), dict(batch=65536),
           dict(table=None), dict(table=66), dict(table_ld=3), dict(table_ld=1 << 41), dict(columns=-1, table_ld=4),
           dict(columns=(1 << 25) + 1, table_ld=1 << 26), dict(free=None), dict(free=65), dict(n_free=-1),
           dict(n_free=1 << 31), dict(taken=None), dict(taken=65), dict(page=0), dict(page=8), dict(page=24),
           dict(page=65552), dict(tokens=-1), dict(tokens=(1 << 29) + 1), dict(slots=None), dict(slots=68),
           dict(positions=None), dict(positions=66), dict(starts=None), dict(starts=66), dict(lengths=None),
           dict(lengths=66), dict(taken_out=None), dict(taken_out=66), dict(taken_out=1024), dict(lengths=64),
           dict(lengths=128), dict(starts=64), dict(starts=128)]
    _refused(mpq, mpq.load().mpq_mx_plan, ok, bad)


ROTATE = dict(Q=64, q_tok=120, q_head=40, K=64, k_tok=80, k_head=40, dtype=1, n=2, heads=3, kv=2, dim=40, positions=64,
              freqs=64, rot=40, interleaved=0, qw=64, kw=64, eps=1e-6, QO=64, qo_tok=120, qo_head=40, KO=64, ko_tok=80,
              ko_head=40, stream=None)


def test_rotate_refusals(mpq):
    lib = mpq.load()
    bad = [dict(Q=None), dict(Q=65), dict(q_tok=-1), dict(q_head=1 << 41), dict(K=None), dict(K=65), dict(k_tok=-1),
           dict(k_head=-1), dict(dtype=3), dict(n=-1), dict(n=1 << 31), dict(heads=0), dict(heads=65536), dict(kv=0),
           dict(kv=65536), dict(dim=0), dict(dim=257), dict(positions=None), dict(positions=66), dict(freqs=None),
           dict(freqs=68), dict(rot=-2), dict(rot=3), dict(rot=42), dict(interleaved=2), dict(interleaved=-1), dict(qw=66),
           dict(kw=66), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(QO=None),
           dict(QO=65), dict(qo_tok=39), dict(qo_head=39), dict(KO=None), dict(KO=65), dict(ko_tok=39), dict(ko_head=39)]
    _refused(mpq, lib.mpq_mx_rotate, ROTATE, bad)
    assert lib.mpq_mx_rotate(*dict(ROTATE, n=0, Q=None, K=None, QO=None, KO=None, positions=None).values()) == 0
    # without a norm eps is not looked at
    assert lib.mpq_mx_rotate(*dict(ROTATE, n=0, qw=None, kw=None, eps=-1.0).values()) == 0


def test_append_refusals(mpq):
    lib = mpq.load()
    good = dict(k_codes=64, v_codes=64, k_scales=64, v_scales=64, n_pages=4, page_size=16, kv_heads=2, head_dim=40, format=1)
    cache = mpq.MXCacheView(*good.values())
    ok = dict(cache=ctypes.addressof(cache), Q=64, q_tok=120, q_head=40, K=64, k_tok=80, k_head=40, V=64, v_tok=80,
              v_head=40, dtype=1, n=2, heads=3, positions=64, slots=64, freqs=64, rot=40, interleaved=0, qw=64, kw=64,
              eps=1e-6, QO=64, qo_tok=120, qo_head=40, stream=None)
    bad = [dict(cache=None), dict(Q=None), dict(Q=65), dict(q_tok=-1), dict(q_head=-1), dict(K=None), dict(K=65),
           dict(k_tok=-1), dict(k_head=-1), dict(V=None), dict(V=65), dict(v_tok=-1), dict(v_head=-1), dict(dtype=-1),
           dict(n=-1), dict(n=1 << 31), dict(heads=0), dict(positions=None), dict(positions=65), dict(slots=None),
           dict(slots=68), dict(freqs=None), dict(freqs=68), dict(rot=41), dict(rot=42), dict(interleaved=2), dict(qw=65),
           dict(kw=65), dict(eps=0.0), dict(QO=None), dict(QO=65), dict(qo_tok=39), dict(qo_head=39)]
    _refused(mpq, lib.mpq_mx_cache_append, ok, bad)
    for kw in (dict(format=2), dict(page_size=8), dict(kv_heads=0), dict(head_dim=257), dict(n_pages=0), dict(k_codes=None),
               dict(v_scales=65)):
        worse = mpq.MXCacheView(*dict(good, **kw).values())
        _refused(mpq, lib.mpq_mx_cache_append, ok, [dict(cache=ctypes.addressof(worse))])
    assert lib.mpq_mx_cache_append(*dict(ok, n=0, Q=None, K=None, V=None, QO=None, slots=None).values()) == 0


def test_route_refusals(mpq):
    lib = mpq.load()
    ok = dict(logits=64, dtype=0, n=3, experts=8, ld=8, k=2, renorm=1, chosen=64, weights=64, order=64, place=64,
              offsets=64, space=None, nbytes=0, stream=None)
    bad = [dict(logits=None), dict(logits=66), dict(dtype=3), dict(n=-1), dict(n=(1 << 20) + 1), dict(experts=0),
           dict(experts=1025, ld=1025), dict(ld=7), dict(k=0), dict(k=9), dict(experts=100, ld=100, k=65), dict(renorm=2),
           dict(chosen=None), dict(chosen=66), dict(weights=None), dict(weights=66), dict(order=None), dict(order=66),
           dict(place=None), dict(place=66), dict(offsets=None), dict(offsets=66), dict(space=68, nbytes=1 << 20),
           dict(n=65, space=64, nbytes=47)]
    _refused(mpq, lib.mpq_mx_route, ok, bad)
    for args in ((-1, 8, 2), (3, 0, 1), (3, 1025, 1), (3, 8, 9), (3, 8, 0)):
        assert lib.mpq_mx_route_workspace(*args) == mpq.MPQ_ERR_INVALID_ARG
    # a byte for every expert and 16 or 64 tokens, and for many tokens their sums; 64 tokens need none
    assert mpq.mx_route_workspace(64, 8, 2) == 0 and mpq.mx_route_workspace(65, 8, 2) == 48
    assert mpq.mx_route_workspace(1 << 20, 8, 2) == 16384 * 8 + 16385 * 8 * 4


EXPERTS = dict(X=64, xt=2, n=30, x_ld=40, wc=64, ws=64, experts=3, c=5, d=40, offsets=64, order=64, m=60, k=2, bias=None,
               Y=64, dtype=1, ld=5, space=None, nbytes=0, stream=None)


def test_experts_refusals(mpq):
    lib = mpq.load()
    bad = [dict(X=None), dict(X=65), dict(xt=5), dict(n=-1), dict(n=(1 << 20) + 1), dict(x_ld=39), dict(wc=None),
           dict(wc=72), dict(ws=None), dict(ws=66), dict(experts=0), dict(experts=1025), dict(c=-1), dict(c=1 << 41, ld=1 << 41),
           dict(d=0), dict(d=4194305, x_ld=4194305), dict(offsets=None), dict(offsets=66), dict(order=66), dict(m=-1),
           dict(m=(1 << 26) + 1), dict(k=0), dict(k=1 << 31), dict(bias=66), dict(Y=None), dict(Y=65), dict(dtype=7),
           dict(ld=4), dict(order=None), dict(order=None, k=1), dict(order=None, m=30), dict(n=0), dict(space=72, nbytes=1 << 20),
           dict(space=64, nbytes=64), dict(n=1 << 20, d=4096, x_ld=4096)]
    _refused(mpq, lib.mpq_mx_experts, EXPERTS, bad)
    assert lib.mpq_mx_experts(*dict(EXPERTS, m=0, Y=None).values()) == 0
    assert lib.mpq_mx_experts(*dict(EXPERTS, c=0, ld=0, wc=None, ws=None, Y=None).values()) == 0
    assert lib.mpq_mx_experts(*dict(EXPERTS, n=0, m=0, X=None, Y=None).values()) == 0
    for args in ((-1, 4, 3, 5, 40), (4, -1, 3, 5, 40), (4, 4, 0, 5, 40), (4, 4, 3, -1, 40), (4, 4, 3, 5, 0),
                 (1 << 20, 4, 3, 5, 4096)):
        assert lib.mpq_mx_experts_workspace(*args) == mpq.MPQ_ERR_INVALID_ARG
    assert mpq.mx_experts_workspace(0, 0, 3, 5, 40) == 0
    # the quantized rows and one of zeros at least
    assert mpq.mx_experts_workspace(30, 60, 3, 5, 40) >= 31 * (64 + 4)


# about every number of tokens at which the work is cut in another way
STEPS = sorted({0, 1 << 20} | {v for t in (1, 2, 4, 5, 16, 64, 256, 1023, 1024, 4096, 8192, 16384, 65472, 65536)
                               for v in (t - 1, t, t + 1)})


EXPERTS_OF_STEPS = [1, 2, 3, 8, 50, 64, 257, 600, 1000, 1024]


@pytest.mark.parametrize("experts", EXPERTS_OF_STEPS)
def test_a_routing_workspace_for_more_tokens_does_for_fewer(mpq, experts):
    """What a server allocates for its longest step holds for every shorter one."""
    for k in sorted({1, min(experts, 8)}):
        sizes = [mpq.mx_route_workspace(n, experts, k) for n in STEPS]
        assert sizes == sorted(sizes), (k, [n for n, a, b in zip(STEPS[1:], sizes, sizes[1:]) if b < a])


@pytest.mark.parametrize("experts", EXPERTS_OF_STEPS)
def test_an_experts_workspace_for_more_rows_does_for_fewer(mpq, experts):
    k = min(experts, 8)
    for c, d in ((256, 256), (1000, 40), (95, 6623), (5632, 512), (2048, 4000)):
        wide = -(-d // 128) * 128
        fits = [n for n in STEPS if n * k <= 1 << 26 and (n + 1) * wide < 1 << 32]
        sizes = [mpq.mx_experts_workspace(n, n * k, experts, c, d) for n in fits]
        assert sizes == sorted(sizes), (c, d, [n for n, a, b in zip(fits[1:], sizes, sizes[1:]) if b < a])
        for n in (1, 3, 4, 5, 300):   # more rows of the same tokens
            sizes = [mpq.mx_experts_workspace(n, m, experts, c, d) for m in STEPS]
            assert sizes == sorted(sizes), (n, c, d, [m for m, a, b in zip(STEPS[1:], sizes, sizes[1:]) if b < a])
        for m in (8, 64, 65, 1000):   # more tokens of as many rows
            sizes = [mpq.mx_experts_workspace(n, m, experts, c, d) for n in fits if n > 0]
            assert sizes == sorted(sizes), (m, c, d)


def test_combine_refusals(mpq):
    lib = mpq.load()
    ok = dict(Y=64, yt=1, m=6, c=5, y_ld=5, place=64, weights=64, n=3, k=2, R=64, r_ld=5, Z=64, dtype=1, ld=5, stream=None)
    bad = [dict(Y=None), dict(Y=65), dict(yt=3), dict(m=-1), dict(m=(1 << 26) + 1), dict(c=-1), dict(c=4194305, y_ld=4194305,
           r_ld=4194305, ld=4194305), dict(y_ld=4), dict(place=None), dict(place=66), dict(weights=None), dict(weights=66),
           dict(n=-1), dict(n=(1 << 20) + 1), dict(k=-1), dict(k=65), dict(R=65), dict(r_ld=4), dict(Z=None), dict(Z=65),
           dict(dtype=9), dict(ld=4)]
    _refused(mpq, lib.mpq_mx_combine, ok, bad)
    assert lib.mpq_mx_combine(*dict(ok, n=0, place=None, weights=None, R=None, Z=None).values()) == 0
    assert lib.mpq_mx_combine(*dict(ok, c=0, y_ld=0, r_ld=0, ld=0).values()) == 0


def test_binding_refuses_host_tensors(mpq):
    import torch
    i = torch.zeros(2, dtype=torch.int32)
    x = torch.zeros(2, 3, 40)
    with pytest.raises(ValueError):
        mpq.mx_plan(i, i, torch.zeros(2, 4, dtype=torch.int32), i, i[:1], 16, 4)
    with pytest.raises(ValueError):
        mpq.mx_rotate(x, x, i, torch.zeros(20, dtype=torch.float64))
    with pytest.raises(ValueError):
        mpq.mx_route(torch.zeros(2, 8), 2)
    with pytest.raises(ValueError):
        mpq.mx_experts(torch.zeros(2, 40), torch.zeros(3, 5, 64, dtype=torch.uint8), torch.zeros(3, 5, 4, dtype=torch.uint8),
                       torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError):
        mpq.mx_combine(torch.zeros(4, 5), torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, 2))


# ------------------------------------------------ the oracle's own sense


def test_plan_by_hand():
    s, p, st, ln, taken, t = ref.plan([5, 16, 0], [1, 2, 17], [[7, -1], [3, -1], [-1, -1]], [9, 1, 2, 4], 1, 16, 22)
    assert s[:3].tolist() == [7 * 16 + 5, 1 * 16, 1 * 16 + 1]
    assert s[3:19].tolist() == list(range(32, 48)) and s[19] == 64 and s[20:].tolist() == [-1, -1]
    assert p[:5].tolist() == [5, 16, 17, 0, 1] and p[20:].tolist() == [0, 0]
    assert st.tolist() == [0, 1, 3, 20] and ln.tolist() == [6, 18, 17] and taken == 4
    assert t.tolist() == [[7, -1], [3, 1], [2, 4]]


def test_route_by_hand():
    c, w, o, p, f = ref.route(np.array([[1.0, 1.0, 0.0], [-np.inf, np.nan, 2.0]]), 2, True)
    assert c.tolist() == [[0, 1], [2, 0]] and w.tolist() == [[0.5, 0.5], [1.0, 0.0]]
    assert o.tolist() == [0, 3, 1, 2] and p.tolist() == [[0, 2], [3, 1]] and f.tolist() == [0, 2, 3, 4]


def test_turn_by_hand():
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    y, _ = ref.turned(x, [1], [np.pi / 2, np.pi], None, 0, False)
    assert np.allclose(y, [[[-3.0, -2.0, 1.0, -4.0, 5.0]]])
    y, _ = ref.turned(x, [1], [np.pi / 2, np.pi], None, 0, True)
    assert np.allclose(y, [[[-2.0, 1.0, -3.0, -4.0, 5.0]]])


# ------------------------------------------------ gathered loads, rings


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    at = tmp_path_factory.mktemp("host")
    so = str(at / "mx_gather.so")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", CSRC,
                           os.path.join(ROOT, "tests", "host", "mx_gather_host.cpp"), "-o", so])
    lib = ctypes.CDLL(so)
    lib.gather_offset.argtypes = [ctypes.c_int64] + [ctypes.c_int] * 4
    lib.gather_offset.restype = ctypes.c_uint32
    return lib


@pytest.mark.parametrize("rows,nb", [(1, 4), (7, 12), (4097, 64), (1023, 65536), (0x7fffffff // (16 * 131072), 131072)])
def test_gathered_loads_stay_inside(host, rows, nb):
    """A live piece of a live stage lies in its row; stages past the row lie
    outside the buffer of (rows + 1) rows, which ends below 2^31."""
    row_bytes, size = 16 * nb, (rows + 0) * 16 * nb
    assert size <= 0x7fffffff
    stages = sorted({0, 1, 2, nb // 8, nb // 4 - 1, nb // 4, nb // 4 + 1, nb // 4 + 3} & set(range(nb // 4 + 4)))
    for row in sorted({0, rows // 2, rows - 1}):
        for lane in range(64):
            piece = (lane % 4) ^ (lane // 16)
            for st in stages:
                at = host.gather_offset(row, lane, row_bytes, st, nb)
                if 4 * st < nb:
                    assert at == row * row_bytes + st * 64 + piece * 16 and at + 16 <= size
                else:
                    assert at >= size
    for lane in range(64):
        for st in stages:
            assert host.gather_offset(-1, lane, row_bytes, st, nb) >= 0x80000000


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    from paper_2002_09049_amd import build as hip
    assert shutil.which(hip.HIPCC), "the HIP compiler builds the library and this listing"
    out = str(tmp_path_factory.mktemp("ring") / "mx_experts.s")
    subprocess.run([hip.HIPCC, *hip.FLAGS, "-I", hip.INCLUDE, "-I", hip.CSRC, "--offload-device-only", "-S",
                    os.path.join(hip.CSRC, "mx_experts.hip"), "-o", out], check=True, capture_output=True)
    return open(out).read()


TILES = [(f"22mx_experts_tile_kernelILi{m}ELi{n}EEEvNS_9MxExpertsE", m + n) for m, n in ((2, 1), (2, 2))]
TILES.append(("22mx_experts_stay_kernelENS_9MxExpertsE", 8))


def _parts(listing, name):
    """The code up to the loop over K, the loop, and what follows it."""
    ops = ring.ops_of(listing, f"_ZN3mpq12_GLOBAL__N_1{name}")
    head, loop = ring.head_and_loop(ops)
    return head, loop, ops[len(head) + len(loop):]


@pytest.mark.parametrize("name,loads", TILES)
def test_the_rings_of_experts_wait(listing, name, loads):
    """As tests/test_mx_ring_cpu.py has it for one matrix: at every barrier the
    stage that it announces has arrived, and the order of loads is fixed."""
    head, loop, _ = _parts(listing, name)
    first = head.index(("lds",))
    # what finds the piece and the gathered rows is loaded, and waited for, before the ring starts
    start = max(i for i, o in enumerate(head[:first]) if o[0] == "pin")
    assert sum(o == ("other",) for o in head[:first]) >= 1 and start < first
    assert loop.count(("lds",)) == 4 * loads and loop.count(("barrier",)) == 4
    assert ring.late_stages(head, loop, loads) == []
    assert ring.mixed_regions(head[start:]) == 0 and ring.mixed_regions(loop) == 0


def test_the_next_tile_starts_with_an_empty_ring(listing):
    """The workgroups that stay: behind the loop everything has landed before the
    next tile's first loads go out, its scales' and three stages; then the code
    in front of the loop runs again.  What else is in flight there (rows' places,
    stores of the sums) can only make a wait that counts from the youngest longer."""
    name, loads = TILES[-1]
    head, loop, tail = _parts(listing, name)
    first = tail.index(("lds",))
    landed = tail.index(("wait", 0))
    assert tail.index(("barrier",)) > landed and first > tail.index(("barrier",))
    assert not any(o in (("lds",), ("other",)) for o in tail[:landed])
    # the first stage; the others follow between the sums' writes, once for every way of writing them
    runs, at = [], 0
    while ("lds",) in tail[at:]:
        start = tail.index(("lds",), at)
        at = start
        while tail[at][0] in ("lds", "pin"):
            at += 1
        runs.append([o for o in tail[start:at] if o == ("lds",)])
    assert all(len(r) in (loads, 2 * loads) for r in runs) and len(runs[0]) == loads and len(runs) > 2
    scales = [o for o in tail[:first] if o == ("other",)][-2:]
    again = max(i for i, o in enumerate(head) if o[0] == "label" and i > max(
        j for j, p in enumerate(head) if p == ("lds",)) and ("barrier",) in head[i:])
    assert head[again:].count(("other",)) >= 2 and ("lds",) not in head[again:]
    assert ring.late_stages(scales + 3 * loads * [("lds",)] + head[again:], loop, loads) == []
    assert ring.mixed_regions(tail[landed:]) == 0
