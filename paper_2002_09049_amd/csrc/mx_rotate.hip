// Norms and rotation of queries' and keys' heads (mpq_mx_rotate), and the same
// with keys and values quantized into the cache (mpq_mx_cache_append).
//
// A head's row: x' = x / sqrt(mean x^2 + eps) w, then each pair (a, b) of its
// first `rot` elements turns by the angle position * freq: (a cos - b sin, b cos +
// a sin).  The angle is found in turns, in 64 bits, and its whole turns are
// dropped before sine and cosine, so a far position costs no accuracy.  They
// are the same for all heads of a token, so a workgroup takes a few tokens with
// all their heads, computes one angle a thread into LDS, and goes through the
// rows: eight elements a thread, 4 ceil(dim / 32) threads a row, rounded up to a
// power of two for the sum of squares; a quad holds a block of the cache.  The
// partner of an element half a head away comes through LDS, a wavefront's part
// each; a row is read whole before it is written, so a call may write in place.
#include "mpq.h"
#include "mx_cache.hpp"

namespace mpq {

namespace {

constexpr int kThreads = 256;
constexpr int kAngles = kThreads;   // of a workgroup

// Of one launch: tokens and heads of a workgroup.
struct Share {
    int tokens, heads, rows;   // rows: heads of all kinds a token has
};

// The sum over the kLanes lanes of a row.
template <int kLanes>
__device__ __forceinline__ float row_sum(float v)
{
    v += xstep<0>(v);
    v += xstep<1>(v);
    if constexpr (kLanes >= 8) v += xstep<2>(v);
    if constexpr (kLanes >= 16) v += xstep<3>(v);
    if constexpr (kLanes >= 32) {
        float a, b;
        swap_step<false>(v, a, b);
        v = a + b;
    }
    return v;
}

// The eight elements at j of a row whose elements lie at `row` in LDS: turned.
__device__ __forceinline__ void turn_halves(float (&x)[8], const float *row, int j, int half, const float *cos,
                                            const float *sin)
{
    if (half % 4 == 0) {   // four neighbours are of one half, their angles aligned
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int at = j + 4 * q;
            if (at >= 2 * half) continue;
            const bool upper = at >= half;
            const int i = upper ? at - half : at;
            const f32x4 c = *(const f32x4 *)(cos + i), s = *(const f32x4 *)(sin + i);
            const f32x4 other = *(const f32x4 *)(row + (upper ? i : at + half));
#pragma unroll
            for (int v = 0; v < 4; ++v) x[4 * q + v] = x[4 * q + v] * c[v] + (upper ? other[v] : -other[v]) * s[v];
        }
    } else {
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            const int at = j + v;
            if (at >= 2 * half) continue;
            const bool upper = at >= half;
            const int i = upper ? at - half : at;
            const float other = row[upper ? i : at + half];
            x[v] = x[v] * cos[i] + (upper ? other : -other) * sin[i];
        }
    }
}

__device__ __forceinline__ void turn_neighbours(float (&x)[8], int j, int half, const float *cos, const float *sin)
{
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int i = j / 2 + v;
        if (i >= half) continue;
        const float a = x[2 * v], b = x[2 * v + 1], c = cos[i], s = sin[i];
        x[2 * v] = a * c - b * s;
        x[2 * v + 1] = b * c + a * s;
    }
}

// kFmt -1: keys go to KO, values are not looked at.
template <int kFmt, int kLanes, class T>
__global__ void __launch_bounds__(kThreads) mx_rotate_kernel(MxRotate r, Share share)
{
    __shared__ __align__(16) float cosines[kAngles], sines[kAngles];
    __shared__ __align__(16) float rows[kThreads * 8];
    const int half = r.rot / 2, pitch = (half + 3) / 4 * 4;
    const int64_t token0 = (int64_t)blockIdx.x * share.tokens;
    const int tokens = (int)min((int64_t)share.tokens, r.n - token0);
    const int head0 = blockIdx.y * share.heads, heads = min(share.heads, share.rows - head0);
    for (int i = threadIdx.x; i < tokens * half; i += kThreads) {
        const int t = i / half, f = i - t * half;
        const double turns = (double)r.positions[token0 + t] * r.freqs[f] * 0.15915494309189533577;
        const double half_turns = 2.0 * (turns - rint(turns));
        // the part that fp32 drops, times the derivative
        const float x = (float)half_turns, rest = (float)(half_turns - (double)x) * 3.14159265f;
        float s, c;
        sincospif(x, &s, &c);
        sines[t * pitch + f] = s + rest * c;
        cosines[t * pitch + f] = c - rest * s;
    }
    __syncthreads();
    const int lane = threadIdx.x % kLanes, j = lane * 8;
    float *row = rows + (threadIdx.x - lane) * 8;
    for (int i = threadIdx.x / kLanes; i < tokens * heads; i += kThreads / kLanes) {
        const int t = i / heads, h = head0 + i - t * heads;
        const int64_t token = token0 + t;
        const bool query = h < r.heads, value = h >= r.heads + r.kv;
        const int head = query ? h : value ? h - r.heads - r.kv : h - r.heads;
        const T *from = query ? (const T *)r.Q + token * r.q_tok + head * r.q_head
                        : value ? (const T *)r.V + token * r.v_tok + head * r.v_head
                                : (const T *)r.K + token * r.k_tok + head * r.k_head;
        const int live = r.dim - j;
        float x[8];
        load8(from + j, live, x);
        if (!value) {
            const float *w = query ? r.qw : r.kw;
            if (w) {
                float sum = 0.0f;
#pragma unroll
                for (int v = 0; v < 8; ++v) sum += x[v] * x[v];
                const float by = 1.0f / sqrtf(row_sum<kLanes>(sum) / (float)r.dim + r.eps);
                float weight[8];
                load8(w + j, live, weight);
#pragma unroll
                for (int v = 0; v < 8; ++v) x[v] = x[v] * by * weight[v];
            }
            if (half > 0) {
                if (r.interleaved) {
                    turn_neighbours(x, j, half, cosines + t * pitch, sines + t * pitch);
                } else {
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    *(f32x4 *)(row + j) = f32x4{x[0], x[1], x[2], x[3]};
                    *(f32x4 *)(row + j + 4) = f32x4{x[4], x[5], x[6], x[7]};
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    turn_halves(x, row, j, half, cosines + t * pitch, sines + t * pitch);
                }
            }
        }
        if (kFmt < 0 || query) {
            T *to = query ? (T *)r.QO + token * r.qo_tok + head * r.qo_head : (T *)r.KO + token * r.ko_tok + head * r.ko_head;
            if (live > 0) store8<false>(to + j, live, x);
        } else {
            constexpr int kF = kFmt < 0 ? kFp4 : kFmt;
            const int64_t slot = r.slots[token];
            if (slot >= 0 && slot < r.c.n_pages * r.c.page && j < r.c.nb * kMxBlock) {
                int64_t page;
                int at;
                find(r.c, slot, page, at);
                const int64_t ph = page * r.c.heads + head, code = code_at<kF>(r.c, ph, at, j), scale = scale_at(r.c, ph, at, j);
                write8<kF>(x, (value ? r.c.v : r.c.k) + code, (value ? r.c.vs : r.c.ks) + scale, j % kMxBlock == 0);
            }
        }
    }
}

template <int kFmt, class T>
hipError_t rotate_lanes(const MxRotate &r, const Share &share, dim3 grid, hipStream_t s)
{
    const int lanes = (r.dim + kMxBlock - 1) / kMxBlock * 4;
    auto kern = lanes <= 4 ? mx_rotate_kernel<kFmt, 4, T> : lanes <= 8 ? mx_rotate_kernel<kFmt, 8, T>
                : lanes <= 16 ? mx_rotate_kernel<kFmt, 16, T> : mx_rotate_kernel<kFmt, 32, T>;
    hipLaunchKernelGGL(kern, grid, dim3(kThreads), 0, s, r, share);
    return hipGetLastError();
}

template <int kFmt>
hipError_t rotate_as(const MxRotate &r, const Share &share, dim3 grid, hipStream_t s)
{
    if (r.dtype == MPQ_F32) return rotate_lanes<kFmt, float>(r, share, grid, s);
    if (r.dtype == MPQ_F16) return rotate_lanes<kFmt, _Float16>(r, share, grid, s);
    return rotate_lanes<kFmt, __bf16>(r, share, grid, s);
}

}  // namespace

hipError_t launch_mx_rotate(const MxRotate &r, bool append, hipStream_t s)
{
    if (r.n <= 0) return hipSuccess;
    Share share;
    share.rows = r.heads + r.kv + (append ? r.kv : 0);
    // an angle a thread: as many tokens as that allows
    const int pitch = (r.rot / 2 + 3) / 4 * 4;
    share.tokens = pitch == 0 ? 4 : max(1, min(8, kThreads / pitch));
    share.heads = share.rows;
    const int64_t blocks = (r.n + share.tokens - 1) / share.tokens;
    const int splits = (share.rows + share.heads - 1) / share.heads;
    if (!launchable(blocks, kThreads) || splits > 65535) return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks, (unsigned)splits);
    LaunchTimer timer(s, append ? "mx_append_kernel" : "mx_rotate_kernel");
    if (!append) return rotate_as<-1>(r, share, grid, s);
    return r.c.fmt == kFp4 ? rotate_as<kFp4>(r, share, grid, s) : rotate_as<kFp8>(r, share, grid, s);
}

}  // namespace mpq
