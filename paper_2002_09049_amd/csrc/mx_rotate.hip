// Norms and rotation of queries' and keys' heads (mpq_mx_rotate), and the same
// with keys and values quantized into the cache (mpq_mx_cache_append).
//
// A head's row: x' = x / sqrt(mean x^2 + eps) w, then each pair (a, b) of its
// first `rot` elements turns by the angle position * freq: (a cos - b sin, b cos +
// a sin).  The angle is found in turns, in 64 bits, and its whole turns are
// dropped before sine and cosine, so a far position costs no accuracy.
//
// A wavefront has one token and some of its heads: it computes the token's
// angles, one a lane, keeps what a lane's eight elements and their partners are
// multiplied by in registers, and goes through the heads, 64 / kLanes at a time, the
// loads of the next ones in flight from the start (the weights' and frequencies',
// waited for first, are issued before them).  A row is kLanes lanes of eight
// elements (4 ceil(dim / 32) rounded up to a power of two, for the sum of
// squares); a quad holds a block of the cache.  The partner of an element half a head
// away comes from the lane half a row away where the whole of a head of 32, 64,
// 128 or 256 turns, else through the wavefront's part of LDS.  A row is read whole
// before it is written, so a call may write in place.  Few tokens are cut into more
// wavefronts, each with its own angles.
//
// fp32 outputs, and keys on their way to the cache, are computed in 64 bits up to
// the one rounding at the end: for a key that is the rounding to its block's
// elements, whose borders a rounding to fp32 before it would cross.
//
// 16384 tokens, 32 + 8 + 8 heads of 128, bf16 with norms into an fp8 cache: 82 to 86
// us, 4.5 TB/s of the 370 MB asked for (inputs partly in the last-level cache), of which
// norms take 2 and what is written into the slots 17 (where the slots follow one
// another it is 93 us, and into an fp4 cache 94); 777 tokens, 7 + 1 heads of 80, fp32:
// 8.1 us; one token, 32 + 8 heads of 128: 4.3 us.
#include <algorithm>
#include <type_traits>

#include "mpq.h"
#include "mx_cache.hpp"

namespace mpq {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;

// The sum over the kLanes lanes of a row.
template <int kLanes, class R>
__device__ __forceinline__ R row_sum(R v)
{
    v += xstep<0>(v);
    v += xstep<1>(v);
    if constexpr (kLanes >= 8) v += xstep<2>(v);
    if constexpr (kLanes >= 16) v += xstep<3>(v);
    if constexpr (kLanes >= 32) {
        R a, b;
        swap_step<false>(v, a, b);
        v = a + b;
    }
    return v;
}

// The value of the lane half a row away.
template <int kLanes>
__device__ __forceinline__ uint32_t half_away(uint32_t v)
{
    if constexpr (kLanes == 4) return dpp<0x4E>(v);              // quad_perm [2,3,0,1]
    else if constexpr (kLanes == 8) return dpp<0x1B>(dpp<0x141>(v));   // row_half_mirror, quad_perm [3,2,1,0]
    else if constexpr (kLanes == 16) return dpp<0x128>(v);       // row_ror:8
    else {
        uint32_t a, b;
        swap_step<false>(v, a, b);
        return threadIdx.x % 32 < 16 ? b : a;
    }
}

// Of a lane's eight elements: the place of each one's partner, and whether it is
// the second of its pair.
struct Pairs {
    int half, j;
    bool interleaved;
    __device__ __forceinline__ bool turns(int v) const { return j + v < 2 * half; }
    __device__ __forceinline__ int angle(int v) const
    {
        const int at = j + v;
        return interleaved ? at / 2 : at < half ? at : at - half;
    }
    __device__ __forceinline__ bool second(int v) const { return interleaved ? v % 2 : j + v >= half; }
    __device__ __forceinline__ int partner(int v) const
    {
        const int at = j + v;
        return at < half ? at + half : at < 2 * half ? at - half : at;
    }
};

// The partners of a row's elements: kSwap by lanes, else (where a head is odd, or
// turns in part) through the wavefront's rows in LDS.
template <int kLanes, bool kSwap, class T>
__device__ __forceinline__ void exchange(const Eight<T> &e, const float (&x)[8], const Pairs &p, float *row, float (&other)[8])
{
    if (p.interleaved) {
#pragma unroll
        for (int v = 0; v < 8; ++v) other[v] = x[v ^ 1];
        return;
    }
    if constexpr (kSwap) {
        Eight<T> o;
#pragma unroll
        for (int i = 0; i < (int)(2 * sizeof(T)); ++i) o.w[i] = half_away<kLanes>(e.w[i]);
        o.values(other);
        return;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    *(f32x4 *)(row + p.j) = f32x4{x[0], x[1], x[2], x[3]};
    *(f32x4 *)(row + p.j + 4) = f32x4{x[4], x[5], x[6], x[7]};
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (p.half % 4 == 0) {   // four neighbours' partners are neighbours
        const f32x4 lo = *(const f32x4 *)(row + p.partner(0)), hi = *(const f32x4 *)(row + p.partner(4));
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            other[v] = lo[v];
            other[v + 4] = hi[v];
        }
    } else {
#pragma unroll
        for (int v = 0; v < 8; ++v) other[v] = row[p.partner(v)];
    }
}

// y to fp32 so that a later rounding to fewer bits is that of y itself: towards
// zero, the last bit set if anything was dropped.
__device__ __forceinline__ float to_odd(double y)
{
    const float f = (float)y;
    uint32_t u = __float_as_uint(f);
    if ((double)f == y || !(fabsf(f) < INFINITY)) return f;
    if (fabs((double)f) > fabs(y)) --u;
    return __uint_as_float(u | 1u);
}

// What a lane's eight elements, and their partners, are multiplied by: weight and
// cosine, the partner's weight and the sine (the first of a pair minus it).
template <class R>
struct Factors {
    R own[8], other[8];

    // weights: of a head, in LDS
    __device__ __forceinline__ void set(bool normed, const float *weights, const Pairs &p, int dim, const double *cosines,
                                        const double *sines)
    {
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            const int at = p.j + v;
            own[v] = normed && at < dim ? (R)weights[at] : (R)1;
            other[v] = (R)0;
            if (!p.turns(v)) continue;
            const R partners = normed ? (R)weights[p.interleaved ? at ^ 1 : p.partner(v)] : (R)1;
            const R s = partners * (R)sines[p.angle(v)];
            own[v] *= (R)cosines[p.angle(v)];
            other[v] = p.second(v) ? s : -s;
        }
    }

    // A row's elements x, normed and turned.
    template <int kLanes, bool kSwap, bool kOdd, class T>
    __device__ __forceinline__ void apply(const Eight<T> &e, float (&x)[8], bool normed, const Pairs &p, float *row,
                                          double inverse_dim, float eps) const
    {
        R by = (R)1;
        if (normed) {
            R sum = (R)0;
#pragma unroll
            for (int v = 0; v < 8; ++v) sum = fma((R)x[v], (R)x[v], sum);
            by = rsqrt(row_sum<kLanes>(sum) * (R)inverse_dim + (R)eps);
        }
        float partner[8];
        if (p.half > 0) exchange<kLanes, kSwap>(e, x, p, row, partner);
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            R y;
            if (kSwap || p.turns(v)) y = fma((R)x[v], own[v], (R)partner[v] * other[v]);
            else y = normed ? (R)x[v] * own[v] : (R)x[v];
            if (normed) y *= by;
            if constexpr (kOdd) x[v] = to_odd(y);
            else x[v] = (float)y;
        }
    }
};

// A lane's rows of one kind, every kStep-th from `lo` below `hi`; the loads of the
// next kDepth are in flight.
template <int kDepth, int kStep, class T>
struct Rows {
    const T *from;
    int64_t stride;
    int lo, hi, live;
    Eight<T> next[kDepth];

    __device__ __forceinline__ void start(const void *base, int64_t offset, int64_t step, int first, int last, int j, int dim)
    {
        from = (const T *)base + offset + j;
        stride = step;
        lo = first;
        hi = last;
        live = dim - j;
#pragma unroll
        for (int i = 0; i < kDepth; ++i)
            if (lo + i * kStep < hi) next[i] = load_eight(from + (lo + i * kStep) * stride, live);
    }
    template <class Body>
    __device__ __forceinline__ void each(Body body)
    {
        for (int h = lo; h < hi; h += kDepth * kStep) {
#pragma unroll
            for (int i = 0; i < kDepth; ++i) {
                const int at = h + i * kStep, more = at + kDepth * kStep;
                if (at >= hi) break;
                const Eight<T> now = next[i];
                if (more < hi) next[i] = load_eight(from + more * stride, live);
                float x[8];
                now.values(x);
                body(at, now, x);
            }
        }
    }
};

// kFmt -1: keys go to KO, values are not looked at.  kMany: the rows of a wavefront
// at a time are of as many tokens, each with all its heads; else of one.
template <int kFmt, int kLanes, bool kSwap, bool kMany, class T>
__global__ void __launch_bounds__(kThreads) mx_rotate_kernel(MxRotate r, int slices, int per)
{
    constexpr int kRows = kWave / kLanes, kDepth = sizeof(T) == 4 ? 2 : 4;
    constexpr int kTokens = kMany ? kRows : 1, kStep = kMany ? 1 : kRows;
    constexpr int kPairs = kTokens * kLanes * 4;   // angles of the wavefront
    constexpr int kTimes = (kPairs + kWave - 1) / kWave;
    using Short = std::conditional_t<std::is_same_v<T, float>, double, float>;
    __shared__ __align__(16) double table[kWaves][2][kPairs];
    __shared__ __align__(16) float weights[kWaves][2][kLanes * 8];
    __shared__ __align__(16) float rows[kWaves][kSwap ? 4 : kWave * 8];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int group = lane / kLanes, j = lane % kLanes * 8, live = r.dim - j;
    const int64_t item = block_of(blockIdx.y) * kWaves + wave, share = quotient(item, slices), token0 = share * kTokens;
    if (token0 >= r.n) return;
    const int64_t token = kMany ? min(token0 + group, r.n - 1) : token0;
    // of the heads of all kinds; none behind the last token
    const int own = kMany ? 0 : group, slice = (int)(item - share * slices) * per, keys = r.heads, values = keys + r.kv;
    const int last = !kMany || token0 + group < r.n ? slice + per : 0;
    const int half = r.rot / 2;
    double *const angles_c = table[wave][0], *const angles_s = table[wave][1];
    const double *cosines = angles_c + (kMany ? group * half : 0), *sines = angles_s + (kMany ? group * half : 0);
    float *row = rows[wave] + (kSwap ? 0 : group * kLanes * 8);
    const Pairs pairs = {half, j, !kSwap && r.interleaved != 0};
    const double inverse_dim = 1.0 / (double)r.dim;

    // angle `lane` and every 64th: of token token0 + angle / half
    double turns[kTimes];
#pragma unroll
    for (int i = 0; i < kTimes; ++i) {
        const int angle = lane + i * kWave;
        turns[i] = 0.0;
        if (angle >= kTokens * half) continue;
        const int t = kMany ? (int)small_quotient((uint32_t)angle, 1.0f / (float)half) : 0;
        turns[i] = (double)r.positions[min(token0 + t, r.n - 1)] * r.freqs[angle - t * half];
    }
    float wq[4], wk[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = lane + i * kWave;
        wq[i] = r.qw && at < r.dim ? r.qw[at] : 0.0f;
        wk[i] = r.kw && at < r.dim ? r.kw[at] : 0.0f;
    }
    int64_t slot = -1;
    if (kFmt >= 0 && slice + per > keys) slot = r.slots[token];
    __builtin_amdgcn_sched_barrier(0);
    Rows<kDepth, kStep, T> q;
    q.start(r.Q, token * r.q_tok, r.q_head, slice + own, min(last, keys), j, r.dim);
    Rows<2, kStep, T> k, v;
    k.start(r.K, token * r.k_tok, r.k_head, max(slice - keys, 0) + own, min(last - keys, r.kv), j, r.dim);
    if constexpr (kFmt >= 0)
        v.start(r.V, token * r.v_tok, r.v_head, max(slice - values, 0) + own, min(last - values, r.kv), j, r.dim);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kTimes; ++i) {
        const int angle = lane + i * kWave;
        if (angle >= kTokens * half) break;
        const double t = turns[i] * 0.15915494309189533577;
        double s, c;
        sincospi(2.0 * (t - rint(t)), &s, &c);
        angles_c[angle] = c;
        angles_s[angle] = s;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = lane + i * kWave;
        if (at >= kLanes * 8) break;
        weights[wave][0][at] = wq[i];
        weights[wave][1][at] = wk[i];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (slice < keys) {
        const bool normed = r.qw != nullptr;
        Factors<Short> f;
        f.set(normed, weights[wave][0], pairs, r.dim, cosines, sines);
        T *to = (T *)r.QO + token * r.qo_tok + j;
        q.each([&](int h, const Eight<T> &e, float (&x)[8]) {
            f.template apply<kLanes, kSwap, false>(e, x, normed, pairs, row, inverse_dim, r.eps);
            if (live > 0) store8<false>(to + h * r.qo_head, live, x);
        });
    }
    if (slice + per <= keys) return;
    const bool normed = r.kw != nullptr;
    if constexpr (kFmt < 0) {
        Factors<Short> f;
        f.set(normed, weights[wave][1], pairs, r.dim, cosines, sines);
        T *to = (T *)r.KO + token * r.ko_tok + j;
        k.each([&](int h, const Eight<T> &e, float (&x)[8]) {
            f.template apply<kLanes, kSwap, false>(e, x, normed, pairs, row, inverse_dim, r.eps);
            if (live > 0) store8<false>(to + h * r.ko_head, live, x);
        });
    } else {
        // (the same in all lanes, and in scalar registers, but with many tokens)
        const bool held = slot >= 0 && slot < r.c.n_pages * r.c.page;
        if (!kMany && !held) return;
        int64_t page = 0;
        int at = 0;
        if (!kMany || held) find(r.c, slot, page, at);
        const auto keep = [&](int h, const float (&x)[8], uint8_t *codes, uint8_t *scales) {
            if ((kMany && !held) || j >= r.c.nb * kMxBlock) return;
            const int64_t ph = page * r.c.heads + h;
            write8<kFmt>(x, codes + code_at<kFmt>(r.c, ph, at, j), scales + scale_at(r.c, ph, at, j), j % kMxBlock == 0);
        };
        v.each([&](int h, const Eight<T> &, const float (&x)[8]) { keep(h, x, r.c.v, r.c.vs); });
        Factors<double> f;
        f.set(normed, weights[wave][1], pairs, r.dim, cosines, sines);
        k.each([&](int h, const Eight<T> &e, float (&x)[8]) {
            f.template apply<kLanes, kSwap, true>(e, x, normed, pairs, row, inverse_dim, r.eps);
            keep(h, x, r.c.k, r.c.ks);
        });
    }
}

template <int kFmt, bool kSwap, bool kMany, class T>
hipError_t rotate_lanes(const MxRotate &r, int lanes, int slices, int per, dim3 grid, hipStream_t s)
{
    auto kern = lanes == 4 ? mx_rotate_kernel<kFmt, 4, kSwap, kMany, T> : lanes == 8 ? mx_rotate_kernel<kFmt, 8, kSwap, kMany, T>
                : lanes == 16 ? mx_rotate_kernel<kFmt, 16, kSwap, kMany, T> : mx_rotate_kernel<kFmt, 32, kSwap, kMany, T>;
    hipLaunchKernelGGL(kern, grid, dim3(kThreads), 0, s, r, slices, per);
    return hipGetLastError();
}

template <int kFmt, class T>
hipError_t rotate_swap(const MxRotate &r, int lanes, bool many, int slices, int per, dim3 grid, hipStream_t s)
{
    const bool swap = !r.interleaved && r.rot == r.dim && r.dim == 8 * lanes;
    if (swap && many) return rotate_lanes<kFmt, true, true, T>(r, lanes, slices, per, grid, s);
    if (swap) return rotate_lanes<kFmt, true, false, T>(r, lanes, slices, per, grid, s);
    if (many) return rotate_lanes<kFmt, false, true, T>(r, lanes, slices, per, grid, s);
    return rotate_lanes<kFmt, false, false, T>(r, lanes, slices, per, grid, s);
}

template <int kFmt>
hipError_t rotate_as(const MxRotate &r, int lanes, bool many, int slices, int per, dim3 grid, hipStream_t s)
{
    if (r.dtype == MPQ_F32) return rotate_swap<kFmt, float>(r, lanes, many, slices, per, grid, s);
    if (r.dtype == MPQ_F16) return rotate_swap<kFmt, _Float16>(r, lanes, many, slices, per, grid, s);
    return rotate_swap<kFmt, __bf16>(r, lanes, many, slices, per, grid, s);
}

}  // namespace

hipError_t launch_mx_rotate(const MxRotate &r, bool append, hipStream_t s)
{
    if (r.n <= 0) return hipSuccess;
    // lanes of a row, and rows that a wavefront has at a time
    const int quads = (r.dim + kMxBlock - 1) / kMxBlock, lanes = quads <= 1 ? 4 : quads <= 2 ? 8 : quads <= 4 ? 16 : 32;
    const int at_once = kWave / lanes, rows = r.heads + r.kv * (append ? 2 : 1);
    // many: where tokens fill the GPU and one has few rows (append, 9 rows of 128 dims,
    // 24480 tokens: 37 us, by a wavefront a token 68; 48 of 32, 5110: 19.5 and 23.7; but
    // 48 of 128, 16384: 89 and 82)
    const bool many = r.n >= 4096 && (rows + at_once - 1) / at_once <= 4;
    const int step = many ? 1 : at_once, passes = (rows + step - 1) / step;
    const int64_t shares = many ? (r.n + at_once - 1) / at_once : r.n;
    // 16 wavefronts a CU
    const int wanted = (int)std::min((int64_t)passes, std::max((int64_t)1, 4096 / shares));
    const int each = (passes + wanted - 1) / wanted, slices = (passes + each - 1) / each;
    const int64_t blocks = (shares * slices + kWaves - 1) / kWaves;
    const dim3 grid(grid_x(blocks), (unsigned)grid_rows(blocks));
    LaunchTimer timer(s, append ? "mx_append_kernel" : "mx_rotate_kernel");
    if (!append) return rotate_as<-1>(r, lanes, many, slices, each * step, grid, s);
    return r.c.fmt == kFp4 ? rotate_as<kFp4>(r, lanes, many, slices, each * step, grid, s)
                           : rotate_as<kFp8>(r, lanes, many, slices, each * step, grid, s);
}

}  // namespace mpq
