// Attention of one new token of every sequence over a paged block-scaled
// cache (mpq_mx_attend):
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q . k_j - m)
// over the tokens j in [max(0, len - window), len), one pass over them with a
// running maximum m and sum.
//
// It is bound by reading the cache, so the work is laid out by what a lane
// can load whole and use where it lands, with no LDS between memory and the
// matrix cores:
//  - The query heads of one cache head (up to 16) are the 16 columns of
//    v_mfma_f32_16x16x32_bf16.  S^T = K Q^T: lane l supplies token l % 16, and
//    as the sum over the head's dimensions may run in any order, its quarter
//    l / 16 of the row, 8 nb consecutive elements.
//  - S^T leaves lane l with column (query head) l % 16 and tokens
//    4 (l / 16) + 0..3 of each 16, which is what O^T = V^T P^T takes as its second
//    operand if the sum over 32 tokens runs in the order that this gives: P
//    never moves between lanes.
//  - For the first operand of O^T lane l loads, for its eight tokens, the eight
//    consecutive dimensions 8 (l % 16) ..; each is converted with its own
//    token's scale, and v_perm pairs tokens.  Output register j then
//    belongs to dimension 8 (row) + j.
// Elements convert to bf16 exactly (at most four significant bits, any
// power of two of a scale).  Q and P are split into bf16 pieces whose sum is
// the value: Q exactly (1 piece for bf16, 2 for f16, 3 for f32), P to 2^-16
// (2 pieces; outputs of 16 bits) or 2^-24 (3).
//
// A long sequence is cut into pieces, one workgroup each, whose four
// wavefronts take 32 tokens in turn; mx_attend_join_kernel joins the pieces.
#include <algorithm>
#include <cmath>

#include "mpq.h"
#include "mx.hpp"

namespace mpq {

namespace {

constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kCols = 16;    // query heads of a workgroup
constexpr int kStep = 32;    // tokens of a step
constexpr float kLn2 = 0.69314718055994531f, kLog2e = 1.4426950408889634f;
// the running maximum follows only a score this far above it (a factor 2^8
// in p, which fp32 sums and bf16 pieces hold as exactly)
constexpr float kSlack = 8.0f;

// Every token of a sequence: [first, len), cut at piece boundaries counted
// from base (a multiple of 16 at or below first).
struct Span {
    int first, len, base;
    __device__ Span(const MxAttend &a, int64_t b)
    {
        const int n = a.lengths[b];
        len = n < 0 ? 0 : n < a.most ? n : a.most;
        first = a.window > 0 && len > a.window ? len - a.window : 0;
        base = first & ~15;
    }
    __device__ int pieces(int piece) const { return (len - base + piece - 1) / piece; }
};

template <class T>
__device__ __forceinline__ void store_as(void *p, int64_t at, float v)
{
    ((T *)p)[at] = (T)v;
}

__device__ __forceinline__ void store_o(void *p, int dtype, int64_t at, float v)
{
    if (dtype == MPQ_F32) store_as<float>(p, at, v);
    else if (dtype == MPQ_F16) store_as<_Float16>(p, at, v);
    else store_as<__bf16>(p, at, v);
}

// Maximum, sum over the four lanes that share a column.
__device__ __forceinline__ float column_max(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}

__device__ __forceinline__ float column_sum(float v)
{
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// Eight elements (fp4: one word, fp8: two) under the scale sc as bf16.
template <int kFmt>
__device__ __forceinline__ void to_bf16(const uint32_t *w, float sc, bf16x2 (&v)[4])
{
    if constexpr (kFmt == kFp4) {
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], sc, 0);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], sc, 1);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], sc, 2);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], sc, 3);
    } else {
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], sc, false);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], sc, true);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], sc, false);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], sc, true);
    }
}

// x as the sum of kPieces bf16 values (each piece the rest's nearest).
template <int kPieces>
__device__ __forceinline__ void split8(const float (&x)[8], bf16x8 (&out)[kPieces])
{
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
    for (int p = 0; p < kPieces; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const __bf16 h = (__bf16)rest[i];
            out[p][i] = h;
            rest[i] -= (float)h;
        }
}

// kWords consecutive words at an address aligned to kAlign bytes.
template <int kWords, int kAlign>
__device__ __forceinline__ void load_words(const uint8_t *p, uint32_t (&w)[kWords])
{
    __builtin_memcpy(w, __builtin_assume_aligned(p, kAlign), sizeof w);
}

template <int kNb, int kFmt>
struct Shape {
    static constexpr int kW = kFmt == kFp4 ? 1 : 2;          // words of eight elements
    static constexpr int kRow = kNb * 16 * kW;               // bytes of a cached row
    static constexpr int kVg = (kNb + 3) / 4;                // groups of 128 dimensions of V
    static constexpr int kDim = kNb * 32;
    static constexpr int kLds = kDim + 4;                    // floats of an LDS row of O
};

// What a lane holds of one step of 32 tokens (two tiles of 16).
template <int kNb, int kFmt>
struct Step {
    using S = Shape<kNb, kFmt>;
    uint32_t k[2][kNb * S::kW];          // its token's quarter row, tile by tile
    uint32_t ks[2][kNb];                 // scale byte of each eight elements
    uint32_t v[2][S::kVg][4][S::kW];     // four tokens of each tile
    uint32_t vs[2][S::kVg];              // their scales, a byte each
};

template <int kNb, int kFmt>
__device__ __forceinline__ void load_step(const MxCacheView &c, int head, const int (&page)[2], const int (&at)[2],
                                          Step<kNb, kFmt> &st)
{
    using S = Shape<kNb, kFmt>;
    const int lane = threadIdx.x % kWave, r = lane % 16, g = lane / 16;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int64_t ph = (int64_t)(page[t] < 0 ? 0 : page[t]) * c.heads + head;
        const int64_t row = ph * c.page + at[t];
        const uint8_t *k = c.k + row * S::kRow + (r * S::kRow + g * (S::kRow / 4));
        load_words<kNb * S::kW, 4 * S::kW * (kNb % 4 == 0 ? 4 / S::kW : kNb % 2 == 0 ? 2 : 1)>(k, st.k[t]);
        const uint8_t *ks = c.ks + ph * kNb * c.page + at[t];
#pragma unroll
        for (int i = 0; i < kNb; ++i) {
            // block of elements 8 (g kNb + i) ..: the same for several i where kNb is even
            constexpr int kSame = kNb % 4 == 0 ? 4 : kNb % 2 == 0 ? 2 : 1;
            if (i % kSame == 0) st.ks[t][i] = ks[(g * kNb + i) / 4 * c.page + r];
            else st.ks[t][i] = st.ks[t][i / kSame * kSame];
        }
#pragma unroll
        for (int q = 0; q < S::kVg; ++q) {
            const int blk = q * 4 + r / 4;     // of the lane's dimensions 128 q + 8 r ..
            if (blk < kNb) {
                const uint8_t *v = c.v + row * S::kRow + (4 * g * S::kRow + (q * 16 + r) * (4 * S::kW));
#pragma unroll
                for (int i = 0; i < 4; ++i) load_words<S::kW, 4 * S::kW>(v + i * S::kRow, st.v[t][q][i]);
                st.vs[t][q] = *(const uint32_t *)(c.vs + (ph * kNb + blk) * c.page + at[t] + 4 * g);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int w = 0; w < S::kW; ++w) st.v[t][q][i][w] = 0;
                st.vs[t][q] = 0;
            }
        }
    }
}

template <int kNb, int kFmt, class T, int kQ, int kP>
__global__ void __launch_bounds__(kThreads) mx_attend_kernel(MxAttend a)
{
    using S = Shape<kNb, kFmt>;
    __shared__ float s_m[kWaves][kCols], s_l[kWaves][kCols];
    __shared__ __align__(16) float s_o[kWaves][kCols * S::kLds];

    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int r = lane % 16, g = lane / 16;
    const int piece = blockIdx.x;
    const int tiles = (a.group + kCols - 1) / kCols;
    const int head = blockIdx.y / tiles, tile = blockIdx.y % tiles;
    const int64_t b = blockIdx.z;
    const int h0 = head * a.group + tile * kCols;                 // first query head
    const int cols = min(kCols, a.group - tile * kCols);
    const Span span(a, b);
    const int begin = span.base + piece * a.piece;
    const int end = min(span.len, begin + a.piece);
    if (a.pieces > 1 && begin >= end) return;   // with one piece, an empty row is written here

    // Q's columns: elements 8 (g kNb + i) .. of head h0 + r
    bf16x8 qf[kNb][kQ];
#pragma unroll
    for (int i = 0; i < kNb; ++i) {
        float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        const int j = 8 * (g * kNb + i);
        if (r < cols) load8((const T *)a.Q + b * a.q_batch + (int64_t)(h0 + r) * a.q_head + j, a.c.dim - j, x);
        split8<kQ>(x, qf[i]);
    }
    const float scale = a.scale * kLog2e;

    float m = -INFINITY, l = 0.0f;   // of column r; l of the lane's own tokens
    f32x4 o[S::kVg][8];
#pragma unroll
    for (int q = 0; q < S::kVg; ++q)
#pragma unroll
        for (int j = 0; j < 8; ++j) o[q][j] = f32x4{0, 0, 0, 0};

    const int steps = begin < end ? (end - begin + kStep - 1) / kStep : 0;
    const int mine = steps > wave ? (steps - wave + kWaves - 1) / kWaves : 0;   // this wavefront's
    int my_page = -1, my_at = 0;
    for (int i = 0; i < mine; ++i) {
        if (i % 32 == 0) {
            // the next 64 tiles' pages, one a lane
            const int tok = begin + kStep * (wave + kWaves * (i + lane / 2)) + 16 * (lane % 2);
            my_page = -1;
            if (tok < end) {
                const int col = tok / a.c.page;
                my_at = tok - col * a.c.page;
                const int pg = a.table[b * a.table_ld + col];
                if (pg >= 0 && pg < a.c.n_pages) my_page = pg;
            }
        }
        const int tok0 = begin + kStep * (wave + kWaves * i);
        int page[2], at[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            page[t] = __builtin_amdgcn_readlane(my_page, 2 * (i % 32) + t);
            at[t] = page[t] < 0 ? 0 : __builtin_amdgcn_readlane(my_at, 2 * (i % 32) + t);
        }
        Step<kNb, kFmt> st;
        load_step<kNb, kFmt>(a.c, head, page, at, st);

        float s[8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4 acc = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < kNb; ++k) {
                union { bf16x2 h[4]; bf16x8 v; } kf;
                to_bf16<kFmt>(&st.k[t][k * S::kW], mx_scale(st.ks[t][k]), kf.h);
#pragma unroll
                for (int p = 0; p < kQ; ++p)
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf.v, qf[k][p], acc, 0, 0, 0);
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) s[4 * t + x] = acc[x] * scale;
        }
        // a step that tokens outside the span, or a page that is not there,
        // touch: their scores are -infinity and their values zeros, whatever
        // the cache holds there
        if (tok0 < span.first || tok0 + kStep > end || page[0] < 0 || page[1] < 0) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int tok = tok0 + 16 * t + 4 * g + x;
                    if (page[t] < 0 || tok < span.first || tok >= end) {
                        s[4 * t + x] = -INFINITY;
#pragma unroll
                        for (int q = 0; q < S::kVg; ++q) {
                            st.vs[t][q] &= ~(255u << (8 * x));
#pragma unroll
                            for (int w = 0; w < S::kW; ++w) st.v[t][q][x][w] = 0;
                        }
                    }
                }
        }
        float top = s[0];
#pragma unroll
        for (int x = 1; x < 8; ++x) top = fmaxf(top, s[x]);
        top = column_max(top);
        if (__any(top > m + kSlack)) {
            const float to = fmaxf(m, top);
            const float f = to == m ? 1.0f : __builtin_amdgcn_exp2f(m - to);   // m = -infinity: 0
            m = to;
            l *= f;
#pragma unroll
            for (int q = 0; q < S::kVg; ++q)
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int x = 0; x < 4; ++x) o[q][j][x] *= f;
        }
        const float base = m == -INFINITY ? 0.0f : m;
        float p[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            p[x] = __builtin_amdgcn_exp2f(s[x] - base);
            l += p[x];
        }
        bf16x8 pf[kP];
        split8<kP>(p, pf);
#pragma unroll
        for (int q = 0; q < S::kVg; ++q) {
            // the eight tokens' eight dimensions as bf16 pairs of dimensions,
            // then as pairs of tokens
            uint32_t d[8][4];
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                bf16x2 h[4];
                to_bf16<kFmt>(st.v[x / 4][q][x % 4], mx_scale((st.vs[x / 4][q] >> (8 * (x % 4))) & 255u), h);
#pragma unroll
                for (int y = 0; y < 4; ++y) d[x][y] = __builtin_bit_cast(uint32_t, h[y]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                union { uint32_t w[4]; bf16x8 v; } vf;
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    vf.w[y] = __builtin_amdgcn_perm(d[2 * y + 1][j / 2], d[2 * y][j / 2],
                                                    j % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int y = 0; y < kP; ++y)
                    o[q][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf.v, pf[y], o[q][j], 0, 0, 0);
            }
        }
    }

    // the wavefronts' results meet in LDS
    l = column_sum(l);
    if (g == 0) {
        s_m[wave][r] = m;
        s_l[wave][r] = l;
    }
#pragma unroll
    for (int q = 0; q < S::kVg; ++q)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int d0 = q * 128 + (4 * g + x) * 8;
            if (d0 < S::kDim) {
                f32x4 lo, hi;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    lo[j] = o[q][j][x];
                    hi[j] = o[q][j + 4][x];
                }
                *(f32x4 *)&s_o[wave][r * S::kLds + d0] = lo;
                *(f32x4 *)&s_o[wave][r * S::kLds + d0 + 4] = hi;
            }
        }
    __syncthreads();
    for (int e = threadIdx.x; e < cols * S::kDim; e += kThreads) {
        const int col = e / S::kDim, d = e % S::kDim;
        float top = s_m[0][col];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_m[w][col]);
        const float base = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f, val = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(s_m[w][col] - base);
            sum += f * s_l[w][col];
            val += f * s_o[w][col * S::kLds + d];
        }
        const int64_t row = b * a.q_heads + h0 + col;
        if (a.pieces > 1) {
            float *out = a.part + (row * a.pieces + piece) * (S::kDim + 2);
            out[2 + d] = val;
            if (d == 0) {
                out[0] = top;
                out[1] = sum;
            }
        } else {
            if (d < a.c.dim)
                store_o(a.O, a.dtype, b * a.o_batch + (int64_t)(h0 + col) * a.o_head + d, sum == 0.0f ? 0.0f : val / sum);
            if (d == 0 && a.lse) a.lse[row] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
        }
    }
}

// Joins the pieces of one query head (a workgroup): thread d sums dimension d.
__global__ void __launch_bounds__(256) mx_attend_join_kernel(MxAttend a)
{
    const int d = threadIdx.x;
    const int64_t b = blockIdx.y, row = b * a.q_heads + blockIdx.x;
    const int dim = a.c.nb * 32;
    const Span span(a, b);
    const int n = span.pieces(a.piece);
    const float *in = a.part + row * a.pieces * (dim + 2);
    float top = -INFINITY;
    for (int i = 0; i < n; ++i) top = fmaxf(top, in[(int64_t)i * (dim + 2)]);
    const float base = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f, val = 0.0f;
    for (int i = 0; i < n; ++i) {
        const float *p = in + (int64_t)i * (dim + 2);
        const float f = __builtin_amdgcn_exp2f(p[0] - base);
        sum += f * p[1];
        if (d < a.c.dim) val += f * p[2 + d];
    }
    if (d < a.c.dim)
        store_o(a.O, a.dtype, b * a.o_batch + (int64_t)blockIdx.x * a.o_head + d, sum == 0.0f ? 0.0f : val / sum);
    if (d == 0 && a.lse) a.lse[row] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <int kNb, int kFmt>
hipError_t launch_shape(const MxAttend &a, dim3 grid, hipStream_t s)
{
    if (a.dtype == MPQ_F32)
        hipLaunchKernelGGL((mx_attend_kernel<kNb, kFmt, float, 3, 3>), grid, dim3(kThreads), 0, s, a);
    else if (a.dtype == MPQ_F16)
        hipLaunchKernelGGL((mx_attend_kernel<kNb, kFmt, _Float16, 2, 2>), grid, dim3(kThreads), 0, s, a);
    else
        hipLaunchKernelGGL((mx_attend_kernel<kNb, kFmt, __bf16, 1, 2>), grid, dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

template <int kFmt>
hipError_t launch_format(const MxAttend &a, dim3 grid, hipStream_t s)
{
    switch (a.c.nb) {
    case 1: return launch_shape<1, kFmt>(a, grid, s);
    case 2: return launch_shape<2, kFmt>(a, grid, s);
    case 3: return launch_shape<3, kFmt>(a, grid, s);
    case 4: return launch_shape<4, kFmt>(a, grid, s);
    case 5: return launch_shape<5, kFmt>(a, grid, s);
    case 6: return launch_shape<6, kFmt>(a, grid, s);
    case 7: return launch_shape<7, kFmt>(a, grid, s);
    case 8: return launch_shape<8, kFmt>(a, grid, s);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace

// A sequence is cut into pieces of a multiple of 128 tokens (a step of each
// wavefront), as many as give every CU a few workgroups.
size_t mx_attend_plan(MxAttend &a)
{
    constexpr int64_t kUnit = kWaves * kStep, kWant = 1024, kMostPieces = 256;
    const int64_t units = a.batch * a.c.heads * ((a.group + kCols - 1) / kCols);
    const int64_t want = std::min(kMostPieces, std::max<int64_t>(1, kWant / std::max<int64_t>(1, units)));
    const int64_t most = a.window > 0 ? std::min<int64_t>(a.most, (int64_t)a.window + 15) : a.most;
    const int64_t piece = std::max(kUnit, ((most + want - 1) / want + kUnit - 1) / kUnit * kUnit);
    a.piece = (int)piece;
    a.pieces = (int)std::max<int64_t>(1, (most + piece - 1) / piece);
    // for any window: pieces is at most want, and at most the tokens' units
    const int64_t bound = std::min(want, (a.most + kUnit - 1) / kUnit);
    return bound <= 1 ? 0 : (size_t)(a.batch * a.q_heads * bound) * (a.c.nb * 32 + 2) * sizeof(float);
}

hipError_t launch_mx_attend(const MxAttend &a, hipStream_t s)
{
    if (a.batch <= 0) return hipSuccess;
    const int64_t gy = (int64_t)a.c.heads * ((a.group + kCols - 1) / kCols);
    if (gy > 65535 || a.batch > 65535) return hipErrorInvalidValue;
    hipError_t e;
    {
        LaunchTimer timer(s, "mx_attend_kernel");
        const dim3 grid((unsigned)a.pieces, (unsigned)gy, (unsigned)a.batch);
        e = a.c.fmt == kFp4 ? launch_format<kFp4>(a, grid, s) : launch_format<kFp8>(a, grid, s);
    }
    if (e != hipSuccess || a.pieces == 1) return e;
    LaunchTimer timer(s, "mx_attend_join_kernel");
    hipLaunchKernelGGL(mx_attend_join_kernel, dim3((unsigned)a.q_heads, (unsigned)a.batch), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace mpq
