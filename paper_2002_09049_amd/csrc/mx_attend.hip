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
//    4 (l / 16) + 0..3, which is what O^T = V^T P^T (v_mfma_f32_16x16x16_bf16)
//    takes as its second operand: P never moves between lanes.
//  - For the first operand of O^T lane l loads, for its four tokens, the eight
//    (heads of up to 64: four) consecutive dimensions 8 (l % 16) ..; each is
//    converted with its own token's scale, and v_perm pairs tokens.  Output
//    register j then belongs to dimension 8 (row) + j.
// Elements convert to bf16 exactly (at most four significant bits), but for fp8
// blocks with a scale byte below 3 (nothing in them reaches 2^-116): theirs
// are rounded to multiples of 2^-133, bf16's least.  Q and P are split into bf16 pieces whose sum is
// the value: Q exactly (1 piece for bf16, 2 for f16, 3 for f32), P to 2^-16
// (2 pieces; outputs of 16 bits) or 2^-24 (3).
//
// A long sequence is cut into pieces, one workgroup each, whose four
// wavefronts take 16 tokens in turn; mx_attend_join_kernel joins the pieces.
//
// One sequence of 131072 tokens, 8 heads of 128 in fp8: 51 us, 5.4 TB/s of the
// 277 MB of cache, and 5 to join; 32 sequences of 1 to 8192 tokens: 63 us, 4.5
// TB/s of 281 MB, and 6.  Forms further from the memory's rate: fp4 (64
// sequences of up to 2048 tokens, 8 heads of 128: 28 us for 72 MB), fp32 queries
// (16 of up to 8192, 4 heads of 128: 20 us for 71 MB; heads of 256, whose
// registers spill, 69 for 142), more than 16 query heads to a cache head, whose
// every 16 read the cache again.
#include <algorithm>
#include <cmath>

#include "mpq.h"
#include "mx.hpp"

namespace mpq {

namespace {

constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kCols = 16;    // query heads of a workgroup
constexpr int kStep = 16;    // tokens of a step
constexpr int kMostPieces = 256;   // of a sequence: one for each thread that joins them
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
    float a, b;
    swap_step<false>(v, a, b);
    swap_step<true>(fmaxf(a, b), a, b);
    return fmaxf(a, b);
}

__device__ __forceinline__ float column_sum(float v)
{
    float a, b;
    swap_step<false>(v, a, b);
    swap_step<true>(a + b, a, b);
    return a + b;
}

// 2 kN elements (four to a word of fp8, eight to one of fp4) under the scale sc
// as bf16.
template <int kFmt, int kN>
__device__ __forceinline__ void to_bf16(const uint32_t *w, float sc, bf16x2 (&v)[kN])
{
    static_assert(kN == 2 || kN == 4, "four or eight elements");
    if constexpr (kFmt == kFp4) {
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], sc, 0);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], sc, 1);
        if constexpr (kN == 4) {
            v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], sc, 2);
            v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], sc, 3);
        }
    } else {
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], sc, false);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], sc, true);
        if constexpr (kN == 4) {
            v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], sc, false);
            v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], sc, true);
        }
    }
}

// x as the sum of kPieces bf16 values (each piece the rest's nearest).  kWide: an
// fp32 value of any size; one whose nearest would be infinity begins with
// bf16's largest, and the next piece has the rest (an infinity's, a NaN's too).
template <int kPieces, bool kWide, int kN, class V>
__device__ __forceinline__ void split(const float (&x)[kN], V (&out)[kPieces])
{
    constexpr float kLargest = 0x1.fep127f;
    float rest[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) rest[i] = x[i];
#pragma unroll
    for (int p = 0; p < kPieces; ++p)
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const __bf16 h = (__bf16)(kWide && p == 0 ? fminf(fmaxf(rest[i], -kLargest), kLargest) : rest[i]);
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
    static constexpr int kE = kNb <= 2 ? 4 : 8;              // dimensions of V a lane holds together
    static constexpr int kVw = kE * kW / 8 > 0 ? kE * kW / 8 : 1;   // their words (fp4, four: half a word)
    static constexpr int kVg = (kNb * 32 + 16 * kE - 1) / (16 * kE);   // groups of 16 kE dimensions
    static constexpr int kDim = kNb * 32;
    static constexpr int kLds = kDim + 4;                    // floats of an LDS row of O
};

// What a lane holds of one step of 16 tokens.
template <int kNb, int kFmt>
struct Step {
    using S = Shape<kNb, kFmt>;
    uint32_t k[kNb * S::kW];         // its token's quarter row
    uint32_t ks[kNb];                // scale byte of each eight elements
    uint32_t v[S::kVg][4][S::kVw];   // four tokens
    uint32_t vs[S::kVg];             // their scales, a byte each
    int page, at;                    // the tokens' page (-1: none) and their place in it
};

template <int kNb, int kFmt>
__device__ __forceinline__ void load_step(const MxCacheView &c, int head, Step<kNb, kFmt> &st)
{
    using S = Shape<kNb, kFmt>;
    const int lane = threadIdx.x % kWave, r = lane % 16, g = lane / 16;
    const int64_t ph = (int64_t)(st.page < 0 ? 0 : st.page) * c.heads + head;
    const int64_t row = ph * c.page + st.at;
    const uint8_t *k = c.k + row * S::kRow + (r * S::kRow + g * (S::kRow / 4));
    load_words<kNb * S::kW, 4 * S::kW * (kNb % 4 == 0 ? 4 / S::kW : kNb % 2 == 0 ? 2 : 1)>(k, st.k);
    const uint8_t *ks = c.ks + ph * kNb * c.page + st.at;
#pragma unroll
    for (int i = 0; i < kNb; ++i) {
        // block of elements 8 (g kNb + i) ..: the same for several i where kNb is even
        constexpr int kSame = kNb % 4 == 0 ? 4 : kNb % 2 == 0 ? 2 : 1;
        if (i % kSame == 0) st.ks[i] = ks[(g * kNb + i) / 4 * c.page + r];
        else st.ks[i] = st.ks[i / kSame * kSame];
    }
#pragma unroll
    for (int q = 0; q < S::kVg; ++q) {
        const int blk = (q * 16 + r) * S::kE / 32;   // of the lane's dimensions kE (16 q + r) ..
        if (blk < kNb) {
            const uint8_t *v = c.v + row * S::kRow + (4 * g * S::kRow + (q * 16 + r) * (S::kE * S::kW / 2));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (S::kE * S::kW < 8) st.v[q][i][0] = *(const uint16_t *)(v + i * S::kRow);
                else load_words<S::kVw, 4 * S::kVw>(v + i * S::kRow, st.v[q][i]);
            }
            st.vs[q] = *(const uint32_t *)(c.vs + (ph * kNb + blk) * c.page + st.at + 4 * g);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int w = 0; w < S::kVw; ++w) st.v[q][i][w] = 0;
            st.vs[q] = 0;
        }
    }
}

template <int kNb, int kFmt, class T, int kQ, int kP>
__global__ void __launch_bounds__(kThreads, kNb > 4 || kQ > 2 ? 2 : 3) mx_attend_kernel(MxAttend a)
{
    using S = Shape<kNb, kFmt>;
    __shared__ float s_m[kWaves][kCols], s_l[kWaves][kCols];
    __shared__ __align__(16) float s_o[kWaves][kCols * S::kLds];

    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane % 16, g = lane / 16;
    const int piece = blockIdx.x;
    const int tiles = (a.group + kCols - 1) / kCols;
    const int head = blockIdx.y / tiles, tile = blockIdx.y % tiles;
    const int64_t b = blockIdx.z;
    const int h0 = head * a.group + tile * kCols;                 // first query head
    const int cols = min(kCols, a.group - tile * kCols);
    // a lane's page of the wavefront's first 64 steps, asked for before
    // the length is known where the span starts at 0
    const int cols_most = a.most / a.c.page;
    int early = -1;
    if (a.window == 0) {
        const int col = (piece * a.piece + kStep * (wave + kWaves * lane)) / a.c.page;
        if (col < cols_most) early = a.table[b * a.table_ld + col];
    }
    const Span span(a, b);
    const int begin = span.base + piece * a.piece;
    const int end = min(span.len, begin + a.piece);
    if (a.pieces > 1 && begin >= end) return;   // with one piece, an empty row is written here

    const float scale = a.scale * kLog2e;

    bf16x8 qf[kNb][kQ];
    float m = -INFINITY, l = 0.0f;   // of column r; l of the lane's own tokens
    f32x4 o[S::kVg][S::kE];
#pragma unroll
    for (int q = 0; q < S::kVg; ++q)
#pragma unroll
        for (int j = 0; j < S::kE; ++j) o[q][j] = f32x4{0, 0, 0, 0};

    const int steps = begin < end ? (end - begin + kStep - 1) / kStep : 0;
    const int mine = steps > wave ? (steps - wave + kWaves - 1) / kWaves : 0;   // this wavefront's
    // step i of this wavefront: its pages, 64 steps' at a time (one a lane), and
    // its part of the cache
    int my_page = -1, my_at = 0;
    const auto fetch = [&](int i, Step<kNb, kFmt> &st) {
        if (i % kWave == 0) {
            const int tok = begin + kStep * (wave + kWaves * (i + lane));
            my_page = -1;
            if (tok < end) {
                const int col = tok / a.c.page;
                my_at = tok - col * a.c.page;
                const int pg = i == 0 && a.window == 0 ? early : a.table[b * a.table_ld + col];
                if (pg >= 0 && pg < a.c.n_pages) my_page = pg;
            }
        }
        st.page = __builtin_amdgcn_readlane(my_page, i % kWave);
        st.at = st.page < 0 ? 0 : __builtin_amdgcn_readlane(my_at, i % kWave);
        load_step<kNb, kFmt>(a.c, head, st);
    };
    const auto attend = [&](int i, Step<kNb, kFmt> &st) {
        const int tok0 = begin + kStep * (wave + kWaves * i);
        f32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < kNb; ++k) {
            union { bf16x2 h[4]; bf16x8 v; } kf;
            to_bf16<kFmt>(&st.k[k * S::kW], mx_scale(st.ks[k]), kf.h);
#pragma unroll
            for (int p = 0; p < kQ; ++p) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf.v, qf[k][p], acc, 0, 0, 0);
        }
        float s[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) s[x] = acc[x] * scale;
        // a step that tokens outside the span, or a page that is not there,
        // touch: their scores are -infinity and their values zeros, whatever
        // the cache holds there
        if (tok0 < span.first || tok0 + kStep > end || st.page < 0) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int tok = tok0 + 4 * g + x;
                if (st.page < 0 || tok < span.first || tok >= end) {
                    s[x] = -INFINITY;
#pragma unroll
                    for (int q = 0; q < S::kVg; ++q) {
                        st.vs[q] &= ~(255u << (8 * x));
#pragma unroll
                        for (int w = 0; w < S::kVw; ++w) st.v[q][x][w] = 0;
                    }
                }
            }
        }
        const float top = column_max(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])));
        if (__any(top > m + kSlack)) {
            const float to = fmaxf(m, top);
            const float f = to == m ? 1.0f : __builtin_amdgcn_exp2f(m - to);   // m = -infinity: 0
            m = to;
            l *= f;
#pragma unroll
            for (int q = 0; q < S::kVg; ++q)
#pragma unroll
                for (int j = 0; j < S::kE; ++j)
#pragma unroll
                    for (int x = 0; x < 4; ++x) o[q][j][x] *= f;
        }
        const float base = m == -INFINITY ? 0.0f : m;
        float p[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            p[x] = __builtin_amdgcn_exp2f(s[x] - base);
            l += p[x];
        }
        bf16x4 pf[kP];
        split<kP, false>(p, pf);
#pragma unroll
        for (int q = 0; q < S::kVg; ++q) {
            // the four tokens' kE dimensions as bf16 pairs of dimensions, then
            // as pairs of tokens
            uint32_t d[4][S::kE / 2];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                bf16x2 h[S::kE / 2];
                to_bf16<kFmt>(st.v[q][x], mx_scale((st.vs[q] >> (8 * x)) & 255u), h);
#pragma unroll
                for (int y = 0; y < S::kE / 2; ++y) d[x][y] = __builtin_bit_cast(uint32_t, h[y]);
            }
#pragma unroll
            for (int j = 0; j < S::kE; ++j) {
                union { uint32_t w[2]; i16x4 v; } vf;
#pragma unroll
                for (int y = 0; y < 2; ++y)
                    vf.w[y] = __builtin_amdgcn_perm(d[2 * y + 1][j / 2], d[2 * y][j / 2],
                                                    j % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int y = 0; y < kP; ++y)
                    o[q][j] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vf.v, __builtin_bit_cast(i16x4, pf[y]), o[q][j],
                                                                        0, 0, 0);
            }
        }
    };
    // the next step's loads are in flight while one is computed
    if (mine > 0) {
        Step<kNb, kFmt> even, odd;
        fetch(0, even);
        // Q's columns: elements 8 (g kNb + i) .. of head h0 + r; columns and
        // elements past the last are zeros.  Whole vectors are all loaded
        // before the first is used (from element 0 where there is none).
        const T *q = (const T *)a.Q + b * a.q_batch + (int64_t)(h0 + (r < cols ? r : 0)) * a.q_head;
        float x[kNb][8];
        if (a.c.dim % 8 == 0) {
#pragma unroll
            for (int i = 0; i < kNb; ++i) {
                const int j = 8 * (g * kNb + i);
                load8(q + (j < a.c.dim ? j : 0), 8, x[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kNb; ++i) load8(q + 8 * (g * kNb + i), a.c.dim - 8 * (g * kNb + i), x[i]);
        }
#pragma unroll
        for (int i = 0; i < kNb; ++i) {
            if (r >= cols || 8 * (g * kNb + i) >= a.c.dim)
#pragma unroll
                for (int y = 0; y < 8; ++y) x[i][y] = 0.0f;
            split<kQ, (kQ > 2)>(x[i], qf[i]);
        }
        int i = 0;
        for (; i + 2 < mine; i += 2) {
            fetch(i + 1, odd);
            attend(i, even);
            fetch(i + 2, even);
            attend(i + 1, odd);
        }
        if (i + 1 < mine) {
            fetch(i + 1, odd);
            attend(i, even);
            attend(i + 1, odd);
        } else {
            attend(i, even);
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
            const int d0 = q * 16 * S::kE + (4 * g + x) * S::kE;
            if (d0 < S::kDim) {
#pragma unroll
                for (int h = 0; h < S::kE; h += 4)
                    *(f32x4 *)&s_o[wave][r * S::kLds + d0 + h] =
                        f32x4{o[q][h][x], o[q][h + 1][x], o[q][h + 2][x], o[q][h + 3][x]};
            }
        }
    __syncthreads();
    // the wavefronts' weights under their common maximum
    if (threadIdx.x < kCols) {
        const int col = threadIdx.x;
        float top = s_m[0][col];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_m[w][col]);
        const float base = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(s_m[w][col] - base);
            sum += f * s_l[w][col];
            s_m[w][col] = f;
        }
        const int64_t row = b * a.q_heads + h0 + col;
        if (col < cols) {
            if (a.pieces > 1)
                ((f32x2 *)(a.part + a.batch * a.q_heads * a.pieces * S::kDim))[row * a.pieces + piece] = f32x2{top, sum};
            else if (a.lse)
                a.lse[row] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
        }
        s_l[0][col] = sum == 0.0f ? 0.0f : 1.0f / sum;
    }
    __syncthreads();
    constexpr int kPer = S::kDim / 4;   // threads a column, four dimensions each
    for (int e = threadIdx.x; e < cols * kPer; e += kThreads) {
        const int col = e / kPer, d = e % kPer * 4;
        f32x4 val = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) val += s_m[w][col] * *(const f32x4 *)&s_o[w][col * S::kLds + d];
        if (a.pieces > 1) {
            *(f32x4 *)&a.part[((b * a.q_heads + h0 + col) * a.pieces + piece) * S::kDim + d] = val;
        } else {
            const int64_t at = b * a.o_batch + (int64_t)(h0 + col) * a.o_head + d;
            const float inv = s_l[0][col];
#pragma unroll
            for (int y = 0; y < 4; ++y)
                if (d + y < a.c.dim) store_o(a.O, a.dtype, at + y, val[y] * inv);
        }
    }
}

// Joins the pieces of one query head (a workgroup): its threads weigh a piece
// each, then groups of dim / 4 threads sum every (256 / (dim / 4))th piece, four
// dimensions a thread, and the groups' sums meet in LDS.
__global__ void __launch_bounds__(kThreads) mx_attend_join_kernel(MxAttend a)
{
    __shared__ float s_w[kMostPieces], s_red[2][kWaves];
    __shared__ f32x4 s_sum[kThreads];
    const int t = threadIdx.x, lane = t % kWave, wave = t / kWave;
    const int64_t b = blockIdx.y, row = b * a.q_heads + blockIdx.x;
    const int dim = a.c.nb * 32;
    const Span span(a, b);
    const int n = span.pieces(a.piece);   // at most a.pieces, at most kMostPieces
    const f32x2 *ml = (const f32x2 *)(a.part + a.batch * a.q_heads * a.pieces * dim) + row * a.pieces;
    const f32x2 mine = t < n ? ml[t] : f32x2{-INFINITY, 0.0f};
    float top = mine[0];
#pragma unroll
    for (int d = 32; d; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
    if (lane == 0) s_red[0][wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_red[0][0], s_red[0][1]), fmaxf(s_red[0][2], s_red[0][3]));
    const float w = __builtin_amdgcn_exp2f(mine[0] - (top == -INFINITY ? 0.0f : top));
    s_w[t] = w;
    float sum = w * mine[1];
#pragma unroll
    for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
    if (lane == 0) s_red[1][wave] = sum;
    __syncthreads();
    sum = (s_red[1][0] + s_red[1][1]) + (s_red[1][2] + s_red[1][3]);

    const int per = dim / 4, groups = kThreads / per, group = t / per;   // threads past groups * per idle
    f32x4 val = {0, 0, 0, 0};
    if (group < groups) {
        const f32x4 *in = (const f32x4 *)(a.part + row * a.pieces * dim) + t % per;
#pragma unroll 4
        for (int i = group; i < n; i += groups) val += s_w[i] * in[(int64_t)i * per];
    }
    s_sum[t] = val;
    __syncthreads();
    if (t < per) {
        for (int i = 1; i < groups; ++i) val += s_sum[i * per + t];
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = 4 * t + i;
            if (d < a.c.dim)
                store_o(a.O, a.dtype, b * a.o_batch + (int64_t)blockIdx.x * a.o_head + d, sum == 0.0f ? 0.0f : val[i] * inv);
        }
    }
    if (t == 0 && a.lse) a.lse[row] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
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

// A sequence is cut into pieces of a multiple of 64 tokens (a step of each
// wavefront), as long as give the three workgroups that fit a CU one each, but
// for several sequences no longer than 960 tokens, which evens out their
// lengths (32 of 1 to 8192 tokens, 8 heads of 128, groups of 8: pieces of 2752,
// 1408, 960, 704 take 74, 70, 62, 65 us).  One sequence's pieces are all alike,
// and two workgroups a CU do (131072 tokens: 51 us and 5 to join them; three: 54
// and 7).  Shorter than 256 tokens, a piece is mostly start and end (16384
// tokens of 8 heads in pieces of 256, 192, 64: 10.6, 12.1, 15.6 us), unless CUs
// would stay empty.  The join costs a launch: up to 512 tokens stay whole (315:
// 7.6 us whole, 5.1 + 4.2 in five pieces; 1000: 13.0 and 4.9 + 4.9), and up to
// 2304 where the heads and sequences alone fill the CUs twice (64 of up to 2048
// tokens, 8 heads in fp4: 27 us whole, 25 + 8.4 in three).  Each rule stands on the
// shapes named, in bf16 and at heads of 128; types and head dimensions whose
// registers allow two workgroups a CU are cut alike.
size_t mx_attend_plan(MxAttend &a)
{
    constexpr int64_t kUnit = kWaves * kStep, kWhole = 512, kWholeFilled = 2304, kCus = 256, kLongest = 960;
    const auto up = [](int64_t n, int64_t d) { return (n + d - 1) / d; };
    const int64_t units = std::max<int64_t>(1, a.batch * a.c.heads * up(a.group, kCols));
    const int64_t want = a.batch == 1 ? 2 * kCus : 3 * kCus;
    // pieces for any window, and so the workspace
    int64_t bound = std::max(up(want, units) + 2, a.batch == 1 ? 0 : up(a.most, kLongest) + 1);
    bound = std::min<int64_t>(std::min<int64_t>(bound, kMostPieces), up(a.most, 128));
    if (a.most <= kWhole || (units >= 2 * kCus && a.most <= kWholeFilled)) bound = 1;
    bound = std::max<int64_t>(1, bound);

    const int64_t most = a.window > 0 ? std::min<int64_t>(a.most, (int64_t)a.window + 15) : a.most;
    int64_t piece = up(most * units, want);
    if (a.batch > 1) piece = std::min(piece, kLongest);
    piece = std::max<int64_t>(piece, units * (most / 256) >= kCus ? 256 : 128);
    if (most <= kWhole || (units >= 2 * kCus && most <= kWholeFilled)) piece = std::max<int64_t>(1, most);
    piece = up(std::max(piece, up(most, bound)), kUnit) * kUnit;
    piece = std::max(piece, kUnit);
    a.piece = (int)piece;
    a.pieces = (int)std::max<int64_t>(1, up(most, piece));
    return bound == 1 ? 0 : (size_t)(a.batch * a.q_heads * bound) * (a.c.nb * 32 + 2) * sizeof(float);
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
