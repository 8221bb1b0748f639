// Products of fp4 rows on the matrix cores' scaled 4-bit instruction:
// v_mfma_scale_f32_16x16x128 takes, from lane l, the 32 elements of one block
// of row l % 16 (16 bytes) and that block's scale byte, so a block's scale costs
// nothing beside its product, and sums 128 products (four blocks, one for each
// l / 16) in fp32.  Rows of W are the instruction's rows, tokens its columns.
//
// The order of the sum is free as long as both operands share it.
//
// Here is what one workgroup does; mx_product.hip has the kernels of one
// matrix W, mx_experts.hip those of rows grouped by expert.
#pragma once

#include <type_traits>

#include "mpq.h"
#include "mx.hpp"
#include "mx_stage.hpp"

namespace mpq {

namespace {

// One lane's share of a chunk (512 elements, 256 bytes) of a row: block 4i + g
// for instruction i, so that the four lanes of a row read 64 consecutive bytes,
// and a word whose byte i is that block's scale.  The row's scales lie
// the other way, 4i .. 4i + 3 in word i: lane g reads word g and the four lanes of
// the row exchange bytes.
typedef uint16_t __attribute__((may_alias)) half_word;
typedef uint32_t __attribute__((may_alias)) word;
typedef uint64_t __attribute__((may_alias)) two_words;

constexpr int kChunkBlocks = 16;
struct Share {
    u32x4 c[4];
    uint32_t s;
};

// Byte i of lane group g's result is byte g of group i's word.
__device__ __forceinline__ uint32_t transpose_bytes(uint32_t w, int g)
{
    uint32_t a, b;
    swap_step<true>(w, a, b);    // groups g % 2 and g % 2 + 2
    w = __builtin_amdgcn_perm(b, a, g / 2 ? 0x07060302u : 0x05040100u);
    swap_step<false>(w, a, b);   // groups g / 2 * 2 and g / 2 * 2 + 1
    return __builtin_amdgcn_perm(b, a, g % 2 ? 0x07030501u : 0x06020400u);
}

// Chunk k / 16 of a row of nb blocks, its scales not yet exchanged.  kWhole: the
// chunk lies inside the row; else blocks past it are zeros.
template <bool kWhole>
__device__ __forceinline__ void load_share(Share &v, const uint8_t *codes, const uint8_t *scales, int64_t row, int nb,
                                           int k, int g)
{
    const uint8_t *p = codes + (row * nb + k + g) * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        v.c[i] = kWhole || k + 4 * i < nb ? *(const u32x4 *)(p + 64 * i) : u32x4{0, 0, 0, 0};
    v.s = kWhole || k + 4 * g < nb ? *(const uint32_t *)(scales + row * nb + k + 4 * g) : 0u;
}

__device__ __forceinline__ i32x8 widen(u32x4 v)
{
    return i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
}

// acc += a b^T over the lanes' blocks i of a chunk (4 in the two format
// operands: E2M1).
template <int kI>
__device__ __forceinline__ f32x4 multiply_block(const Share &a, const Share &b, f32x4 acc)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(widen(a.c[kI]), widen(b.c[kI]), acc, 4, 4, kI, (int)a.s,
                                                            kI, (int)b.s);
}

__device__ __forceinline__ f32x4 multiply_chunk(const Share &a, const Share &b, f32x4 acc)
{
    acc = multiply_block<0>(a, b, acc);
    acc = multiply_block<1>(a, b, acc);
    acc = multiply_block<2>(a, b, acc);
    return multiply_block<3>(a, b, acc);
}

__device__ __forceinline__ void store_y(void *Y, int dtype, int64_t at, float v)
{
    if (dtype == MPQ_F32) ((float *)Y)[at] = v;
    else if (dtype == MPQ_F16) ((_Float16 *)Y)[at] = (_Float16)v;
    else ((__bf16 *)Y)[at] = (__bf16)v;
}

// Few tokens: a workgroup owns 16 rows of W and 16 kNT tokens; its wavefronts
// take the chunks of K in turn, straight from memory to registers, and their
// sums meet in LDS, added in wavefront order.  At 16 tokens, 4096 x 4096, 4.5
// us; more are bound by the vector cache, which serves the lanes of a load of
// 16-byte pieces one after another (64, 25088 x 4096: 34 us, 1.6 TB/s of W).
constexpr int kFewWaves = 8;

// A workgroup may have more than 16 rows of W: kSplit of its wavefronts then take
// the chunks of the same 16 in turn, and the next kSplit the next 16 rows.
template <int kSplit>
constexpr int kFewRows = kFewWaves / kSplit * 16;

// The sums of a workgroup's wavefronts to Y.
template <int kNT, int kSplit>
__device__ __forceinline__ void join_waves(const MxProduct &p, float (&part)[kFewWaves][kNT][kWave * 4],
                                           const f32x4 (&acc)[kNT], int64_t c0, int64_t t0)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
#pragma unroll
    for (int t = 0; t < kNT; ++t) *(f32x4 *)&part[wave][t][lane * 4] = acc[t];
    __syncthreads();
    // output o of the tile: row o % kRows of W, token o / kRows; lane l's register i
    // holds row 4 (l / 16) + i of the wavefront's 16, token l % 16
    constexpr int kRows = kFewRows<kSplit>;
    for (int o = threadIdx.x; o < kNT * 16 * kRows; o += kFewWaves * kWave) {
        const int row = o % kRows, tok = o / kRows;
        const int at = ((row % 16 / 4) * 16 + tok % 16) * 4 + row % 4;
        if (c0 + row >= p.c || t0 + tok >= p.n) continue;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kSplit; ++w) v += part[row / 16 * kSplit + w][tok / 16][at];
        if (p.bias) v += p.bias[c0 + row];
        store_y(p.Y, p.dtype, (t0 + tok) * p.ldy + c0 + row, v);
    }
}

// The workgroup of rows c0 .. of W and tokens t0 .. (up to p.n); row_of gives a
// token's row of X.
template <int kNT, int kSplit, class RowOf>
__device__ __forceinline__ void few_product(const MxProduct &p, int64_t c0, int64_t t0, RowOf row_of)
{
    __shared__ __align__(16) float part[kFewWaves][kNT][kWave * 4];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane % 16, g = lane / 16;
    const int nb = p.nb;
    // rows past the end repeat the last one: their sums are not stored
    const int64_t wrow = min(c0 + wave / kSplit * 16 + r, p.c - 1);
    int64_t xrow[kNT];
    f32x4 acc[kNT];
#pragma unroll
    for (int t = 0; t < kNT; ++t) {
        xrow[t] = row_of(min(t0 + 16 * t + r, p.n - 1));
        acc[t] = f32x4{0, 0, 0, 0};
    }
    const auto chunk = [&](auto whole, int k) {
        Share a, b[kNT];
        load_share<decltype(whole)::value>(a, p.wc, p.ws, wrow, nb, k, g);
#pragma unroll
        for (int t = 0; t < kNT; ++t) load_share<decltype(whole)::value>(b[t], p.xc, p.xs, xrow[t], nb, k, g);
        a.s = transpose_bytes(a.s, g);
#pragma unroll
        for (int t = 0; t < kNT; ++t) {
            b[t].s = transpose_bytes(b[t].s, g);
            acc[t] = multiply_chunk(a, b[t], acc[t]);
        }
    };
    int k = wave % kSplit * kChunkBlocks;
    for (; k + kChunkBlocks <= nb; k += kSplit * kChunkBlocks) chunk(std::true_type(), k);
    if (k < nb) chunk(std::false_type(), k);   // the chunk that the row ends in
    join_waves<kNT, kSplit>(p, part, acc, c0, t0);
}

// One to kN tokens, quantized on the way: a wavefront quantizes its chunk of
// every token itself (eight elements a lane, a block a quad, as
// mx_quantize.hip), through a part of LDS of its own, so the call is one
// launch and X is read by each workgroup.  4096 x 4096, one token: 4.0 us,
// against 1.9 + 3.8 in two launches (and their gap); four tokens, 25088 x 4096:
// 14 us, 3.9 TB/s of W.  With more than four tokens the quantization in every
// workgroup costs more than the launch.
//
// The workgroup of rows c0 .. of W and the n tokens t0 ..; at gives the start of
// a token's row of X, none whether it is zeros instead.
template <int kN, int kSplit, class T, class At, class None>
__device__ __forceinline__ void token_product(const MxProduct &p, int64_t c0, int64_t t0, int n, int d, At at, None none)
{
    __shared__ __align__(16) float part[kFewWaves][1][kWave * 4];
    __shared__ __align__(16) uint32_t xcodes[kFewWaves][kN][kWave];   // a chunk's codes, eight elements a word
    __shared__ __align__(4) uint8_t xscales[kFewWaves][kN][kChunkBlocks];          // block 4i + g at 4g + i
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane % 16, g = lane / 16;
    const int nb = p.nb;
    const int64_t wrow = min(c0 + wave / kSplit * 16 + r, p.c - 1);
    f32x4 acc[1] = {f32x4{0, 0, 0, 0}};
    struct Chunk {
        Share a;
        Eight<T> x[kN];
    };
    const auto fetch = [&](auto whole, int k, Chunk &c) {
        constexpr bool kWhole = decltype(whole)::value;
        load_share<kWhole>(c.a, p.wc, p.ws, wrow, nb, k, g);
        const int e = k * kMxBlock + 8 * lane;
#pragma unroll
        for (int t = 0; t < kN; ++t) {
            const int token = t < n ? t : 0;
            c.x[t] = load_eight(at(token) + e, none(token) ? 0 : kWhole ? 8 : d - e);
        }
    };
    const auto multiply = [&](Chunk &c) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int t = 0; t < kN; ++t) {
            float x[8];
            c.x[t].values(x);
            const uint32_t s = mx_scale_byte<kFp4>(quad_max(largest_bits(x)));
            uint32_t w[1];
            mx_codes<kFp4>(x, s, w);
            xcodes[wave][t][lane] = w[0];
            const int blk = lane / 4;
            if (lane % 4 == 0) xscales[wave][t][blk % 4 * 4 + blk / 4] = (uint8_t)s;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const bool live = r < kN && r < n;
        Share b;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            b.c[i] = live ? *(const u32x4 *)&xcodes[wave][r][(4 * i + g) * 4] : u32x4{0, 0, 0, 0};
        b.s = live ? *(const word *)&xscales[wave][r][4 * g] : 0u;
        c.a.s = transpose_bytes(c.a.s, g);
        acc[0] = multiply_chunk(c.a, b, acc[0]);
    };
    // this wavefront's chunks inside the rows of X, the next one's loads in
    // flight, then the one that they end in
    constexpr int kTurn = kSplit * kChunkBlocks;
    const int inside = d / kMxBlock;   // whole blocks
    int k = wave % kSplit * kChunkBlocks;
    const int mine = k + kChunkBlocks <= inside ? (inside - kChunkBlocks - k) / kTurn + 1 : 0;
    Chunk even, odd;
    if (mine > 0) {
        const std::true_type whole;
        fetch(whole, k, even);
        int i = 0;
        for (; i + 2 < mine; i += 2, k += 2 * kTurn) {
            fetch(whole, k + kTurn, odd);
            multiply(even);
            fetch(whole, k + 2 * kTurn, even);
            multiply(odd);
        }
        if (i + 1 < mine) {
            fetch(whole, k + kTurn, odd);
            multiply(even);
            multiply(odd);
            k += kTurn;
        } else {
            multiply(even);
        }
        k += kTurn;
    }
    if (k < nb) {
        fetch(std::false_type(), k, even);
        multiply(even);
    }
    join_waves<1, kSplit>(p, part, acc, c0, t0);
}

// Many tokens: a workgroup owns 64 kTM rows of W by 64 kTN tokens, its four
// wavefronts a quarter each (32 kTM by 32 kTN, in v_mfma_scale_f32_32x32x64
// tiles: lane l supplies the 32 elements of one block of row l % 32).
//
// K runs in stages of 128 elements, 64 bytes of every row, in a ring of four
// LDS buffers that loads fill without passing through registers.  While
// stage s is multiplied, the loads of stage s + 3 go out between its products
// (a wavefront has its SIMD to itself, so a load that waits for its turn
// would hold up the matrix core), and the operands of each step are read from LDS
// during the step before, those of stage s + 1 too: the barrier at stage s
// says that stage s + 1 is there.  Stages past the row are zeros: their loads
// lie past the buffer, and every wait counts the same number of loads.
//
// 16-byte piece q of row r lies in place q ^ (r / 4 % 4) of its LDS row, so that
// lanes that read one piece of consecutive rows spread over the banks.  Lanes of
// half h = l / 32 take pieces 2h and 2h + 1, one for each of a stage's two
// steps, so the scales of a lane's row come as a half-word whose bytes the
// steps select.  Scales go to LDS four stages at a time, 16 bytes of a row
// through the registers of a thread: one row's scales lie in one line of
// memory, apart from the other rows', so they are fetched as rarely as
// possible.
//
// 8192 tokens, 4096 x 4096, in 256 by 256 tiles: 81 us, 3.4 PFLOP/s.  The matrix
// cores are busy 47% of a wavefront's cycles; the rest is a tile's start and
// end, which nothing covers (one workgroup a CU), and what the reads of LDS
// and the barriers leave uncovered.

// (the arguments are the same in every lane: a descriptor in scalar registers)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const uint8_t *base, int64_t bytes)
{
    const uint64_t at = (uint64_t)base;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)at), hi = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32));
    return __builtin_amdgcn_make_buffer_rsrc((void *)((uint64_t)hi << 32 | lo), (short)0,
                                             __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000);
}

// 16 rows' part of a stage into LDS (the 64 lanes' 16 bytes land one after the
// other).  The whole offset is the lane's own: the check against the buffer's
// length is documented to cover that one, not the scalar offset.
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t from, uint8_t *to, uint32_t at)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, to, 16, at, 0, 0, 0);
}

__device__ __forceinline__ u32x4 load_scales(__amdgpu_buffer_rsrc_t from, uint32_t at)
{
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from, at, 0, 0));
}

// acc += a b^T over the lanes' blocks; byte kA of as and byte kB of bs are
// their scales.
template <int kA, int kB>
__device__ __forceinline__ f32x16 multiply_tile(u32x4 a, uint32_t as, u32x4 b, uint32_t bs, f32x16 acc)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(widen(a), widen(b), acc, 4, 4, kA, (int)as, kB, (int)bs);
}

// The compiler moves no access across (no instruction).  The rings' waits count
// loads in the order that they are issued, those into LDS and the scales' into
// registers alike, so between loads of the two kinds stands a pin:
// tests/test_mx_ring_cpu.py reads it off the code that the compiler makes.
__device__ __forceinline__ void pin()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_sched_barrier(0);
}

// A barrier that leaves this wavefront's last kLeft loads in flight
// (__syncthreads would wait for them all); its LDS reads and writes and its
// loads before those are done.
template <int kLeft>
__device__ __forceinline__ void meet()
{
    constexpr int kVmcnt = (kLeft & 15) | (kLeft >> 4) << 14;
    pin();
    __builtin_amdgcn_s_waitcnt(0x0070 | kVmcnt);   // vmcnt(kLeft), lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    pin();
}

// The operands of one step of a stage (64 elements): the lane's pieces of the
// wavefront's rows of W, which start at row wm of the stage, and of its
// tokens, at row 64 kTM + wn.
template <int kTM, int kTN>
struct Operands {
    u32x4 a[kTM], b[kTN];
    // those of row tile i: W's, and the tokens' where there is one
    __device__ __forceinline__ void read(int i, const uint8_t *stage, int step, int wm, int wn, int r, int h)
    {
        const int at = ((2 * h + step) ^ (r / 4 % 4)) * 16;
        a[i] = *(const u32x4 *)(stage + (wm + 32 * i + r) * kStageBytes + at);
        if (i < kTN) b[i] = *(const u32x4 *)(stage + (64 * kTM + wn + 32 * i + r) * kStageBytes + at);
    }
    // one of the two: W's, the tokens'
    template <bool kTokens>
    __device__ __forceinline__ void read_one(int i, const uint8_t *stage, int step, int wm, int wn, int r, int h)
    {
        const int at = ((2 * h + step) ^ (r / 4 % 4)) * 16;
        if constexpr (kTokens) b[i] = *(const u32x4 *)(stage + (64 * kTM + wn + 32 * i + r) * kStageBytes + at);
        else a[i] = *(const u32x4 *)(stage + (wm + 32 * i + r) * kStageBytes + at);
    }
};

// The scales of the lane's rows for one stage, two bytes (a step each) a row
// tile: they lie side by side in LDS, [h][r][tile], and the products select
// their bytes.
// kT half-words, aligned to their size (plain loads: the compiler keeps track
// of which LDS array they read)
template <int kT>
__device__ __forceinline__ void read_scales(const uint8_t *at, uint32_t (&w)[(kT + 1) / 2])
{
    if constexpr (kT == 1) w[0] = *(const half_word *)at;
    else if constexpr (kT == 2) w[0] = *(const word *)at;
    else {
        static_assert(kT == 4, "");
        const uint64_t v = *(const two_words *)at;
        w[0] = (uint32_t)v;
        w[1] = (uint32_t)(v >> 32);
    }
}

template <int kTM, int kTN>
struct Scales {
    uint32_t a[(kTM + 1) / 2], b[(kTN + 1) / 2];
    __device__ __forceinline__ void read(const uint8_t *stage, int wm, int wn, int r, int h)
    {
        const uint8_t *at = stage + h * 512 * ((64 * (kTM + kTN) + 255) / 256);
        read_scales<kTM>(at + 2 * (wm + r * kTM), a);
        read_scales<kTN>(at + 2 * (64 * kTM + wn + r * kTN), b);
    }
};

// Product of row tiles i and j of a step kS.
template <int kS, int kTM, int kTN>
__device__ __forceinline__ f32x16 multiply_pair(const Operands<kTM, kTN> &o, const Scales<kTM, kTN> &sc, int i, int j, f32x16 acc)
{
    // byte of the word: the odd tile's pair is its upper half
    if (i % 2 == 0 && j % 2 == 0) return multiply_tile<kS, kS>(o.a[i], sc.a[i / 2], o.b[j], sc.b[j / 2], acc);
    if (i % 2 == 0) return multiply_tile<kS, kS + 2>(o.a[i], sc.a[i / 2], o.b[j], sc.b[j / 2], acc);
    if (j % 2 == 0) return multiply_tile<kS + 2, kS>(o.a[i], sc.a[i / 2], o.b[j], sc.b[j / 2], acc);
    return multiply_tile<kS + 2, kS + 2>(o.a[i], sc.a[i / 2], o.b[j], sc.b[j / 2], acc);
}

// The products of one step; after(i) runs behind those of row tile i.
template <int kS, int kTM, int kTN, class After>
__device__ __forceinline__ void multiply_operands(const Operands<kTM, kTN> &o, const Scales<kTM, kTN> &sc,
                                                  f32x16 (&acc)[kTM][kTN], After after)
{
#pragma unroll
    for (int i = 0; i < kTM; ++i) {
#pragma unroll
        for (int j = 0; j < kTN; ++j) acc[i][j] = multiply_pair<kS>(o, sc, i, j, acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
        after(i);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// The same with after(i, j) behind each product: what it issues has the time of one
// product, so that little work behind every one hides where much behind every
// fourth does not (a stage of 256 by 256 tiles 1530 cycles, so 1440; its 32 products
// take 1024).
template <int kS, int kTM, int kTN, class After>
__device__ __forceinline__ void multiply_spread(const Operands<kTM, kTN> &o, const Scales<kTM, kTN> &sc,
                                                f32x16 (&acc)[kTM][kTN], After after)
{
#pragma unroll
    for (int i = 0; i < kTM; ++i)
#pragma unroll
        for (int j = 0; j < kTN; ++j) {
            acc[i][j] = multiply_pair<kS>(o, sc, i, j, acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
            after(i, j);
            __builtin_amdgcn_sched_barrier(0);
        }
}

// The sums to Y.  Register v of a tile is row 8 (v / 4) + 4 h + v % 4 of W, token
// r: a wavefront turns two by two tiles (64 rows of W by 64 tokens; 32 where it
// has one tile of them) at a time in its part of LDS, so that a lane then holds
// eight consecutive values of a token's row and eight lanes store 64 of them, a
// whole line of 16-bit values (32 at a time, half a line: 1.5 times the bytes
// written).  The loop over tokens stays rolled: unrolled, with the sums'
// registers as its operands, it took 14 us of a 256 by 256 tile, instruction
// fetches.
//
// A token's row in LDS is 16 pieces of four values; piece q of token t lies in
// place q ^ (t % 16).
constexpr int kTurnRow = 64;   // floats

// Of the tokens lane / 8, + 8, .. below `tokens`: eight values, with the bias
// added, to rows of Y from `to` on; whole: all lanes' eight values are inside
// the rows.
template <class T>
__device__ __forceinline__ void write_turn(T *to, int64_t step, const float *turn, int lane, int tokens, bool whole,
                                           int live, const float (&bias)[8])
{
    const auto one = [&](int t, int inside) {
        const int piece = (lane % 8 * 2) ^ (t % 16);
        const float *row = turn + t * kTurnRow;
        const f32x4 lo = *(const f32x4 *)(row + piece * 4), hi = *(const f32x4 *)(row + (piece ^ 1) * 4);
        float y[8];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            y[v] = lo[v] + bias[v];
            y[v + 4] = hi[v] + bias[v + 4];
        }
        store8<false>(to, inside, y);
        to += step;
    };
    if (whole) {
#pragma unroll 4
        for (int t = lane / 8; t < tokens; t += 8) one(t, 8);
    } else {
#pragma unroll 1
        for (int t = lane / 8; t < tokens; t += 8) one(t, live);
    }
}

template <int kTM, int kTN, int kJ = kTN < 2 ? 1 : 2>   // kJ: token tiles of a turn
__device__ __forceinline__ void write_tiles(const MxProduct &p, float *turn, int64_t c0, int64_t t0, int lane,
                                            const f32x16 (&acc)[kTM][kTN])
{
    const int r = lane % 32, h = lane / 32;
#pragma unroll
    for (int i = 0; i < kTM; i += 2) {
        const bool whole = c0 + 32 * i + 64 <= p.c;
        const int64_t row = c0 + 32 * i + lane % 8 * 8;
        const int live = (int)min((int64_t)8, p.c - row);
        float bias[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (p.bias) load8(p.bias + row, live, bias);
#pragma unroll
        for (int j = 0; j < kTN; j += kJ) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int y = 0; y < kJ; ++y)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x16 &t = acc[i + x][j + y];
                        *(f32x4 *)&turn[(32 * y + r) * kTurnRow + ((8 * x + 2 * q + h) ^ (r % 16)) * 4] =
                            f32x4{t[4 * q], t[4 * q + 1], t[4 * q + 2], t[4 * q + 3]};
                    }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const int64_t first = t0 + 32 * j, at = (first + lane / 8) * p.ldy + row;
            const int tokens = (int)min((int64_t)(32 * kJ), p.n - first);
            if (p.dtype == MPQ_F32) write_turn((float *)p.Y + at, 8 * p.ldy, turn, lane, tokens, whole, live, bias);
            else if (p.dtype == MPQ_F16) write_turn((_Float16 *)p.Y + at, 8 * p.ldy, turn, lane, tokens, whole, live, bias);
            else write_turn((__bf16 *)p.Y + at, 8 * p.ldy, turn, lane, tokens, whole, live, bias);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
}

// The same for 16-bit values, which are rounded on their way into LDS, so that the
// whole of a wavefront's rows of W, 32 kTM, is there of 32 tokens at a time: half
// the bytes through LDS, and a token's 128 or 256 bytes in one store, its reads
// all ahead of it.  Piece q of a token (eight values) lies in place q ^ (token %
// 16), of 64 rows q ^ (token / 2 % 8).  bias: of the wavefront's rows, in LDS;
// between(j) runs while the reads of token tile j are on their way.
template <class T>
__device__ __forceinline__ uint32_t packed_pair(float a, float b)
{
    typedef T two __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), two));
}

template <bool kBias, int kTM, int kTN, class T, class Between>
__device__ __forceinline__ void write_packed(const MxProduct &p, uint8_t *turn, const float *bias, int64_t c0, int64_t t0,
                                             int lane, const f32x16 (&acc)[kTM][kTN], Between between)
{
    constexpr int kPieces = 4 * kTM, kTokens = kWave / kPieces, kTimes = 32 / kTokens;   // of a token; of one load
    const int r = lane % 32, h = lane / 32;
    const auto place = [](int token, int piece) {
        return (token * kPieces + (piece ^ (kTM == 4 ? token % 16 : token / 2 % 8))) * 16;
    };
    const int piece = lane % kPieces, token = lane / kPieces;
    const int64_t row = c0 + 8 * piece;
    const int live = (int)min((int64_t)8, p.c - row);
    const bool rows_live = c0 + 32 * kTM <= p.c;
#pragma unroll
    for (int j = 0; j < kTN; ++j) {
#pragma unroll
        for (int i = 0; i < kTM; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x16 &t = acc[i][j];
                f32x4 y = f32x4{t[4 * q], t[4 * q + 1], t[4 * q + 2], t[4 * q + 3]};
                if constexpr (kBias) y += *(const f32x4 *)(bias + 32 * i + 8 * q + 4 * h);
                *(two_words *)(turn + place(r, 4 * i + q) + 8 * h) =
                    (uint64_t)packed_pair<T>(y[2], y[3]) << 32 | packed_pair<T>(y[0], y[1]);
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        u32x4 out[kTimes];
#pragma unroll
        for (int k = 0; k < kTimes; ++k) out[k] = *(const u32x4 *)(turn + place(token + k * kTokens, piece));
        between(j);
        const int64_t first = t0 + 32 * j;
        const int tokens = (int)min((int64_t)32, p.n - first);
        T *to = (T *)p.Y + (first + token) * p.ldy + row;
        if (rows_live && tokens == 32) {
#pragma unroll
            for (int k = 0; k < kTimes; ++k) *(loose_vector *)(to + k * kTokens * p.ldy) = out[k];
        } else {
#pragma unroll
            for (int k = 0; k < kTimes; ++k) {
                T v[8];
                __builtin_memcpy(v, &out[k], 16);
#pragma unroll
                for (int x = 0; x < 8; ++x)
                    if (token + k * kTokens < tokens && x < live) to[k * kTokens * p.ldy + x] = v[x];
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// A wavefront's sums to Y: 32 kTM rows of W from c0, 32 kTN tokens from t0.
// bias: those of the rows lane kTM / 2, + 1 (loaded_bias); bias_at: room for 32 kTM.
template <int kTM>
struct Bias {
    float of[kTM / 2];
};
template <int kTM>
__device__ __forceinline__ Bias<kTM> loaded_bias(const MxProduct &p, int64_t c0, int lane)
{
    Bias<kTM> b;
#pragma unroll
    for (int i = 0; i < kTM / 2; ++i) {
        const int64_t row = c0 + lane * (kTM / 2) + i;
        b.of[i] = p.bias && row < p.c ? p.bias[row] : 0.0f;
    }
    return b;
}
template <int kTM, int kTN, class Between>
__device__ __forceinline__ void write_sums(const MxProduct &p, uint8_t *turn, float *bias_at, const Bias<kTM> &bias,
                                           int64_t c0, int64_t t0, int lane, const f32x16 (&acc)[kTM][kTN], Between between)
{
    if (p.dtype == MPQ_F32) {
#pragma unroll
        for (int j = 0; j < kTN; ++j) between(j);
        write_tiles<kTM, kTN, 1>(p, (float *)turn, c0, t0, lane, acc);
        return;
    }
    if (p.bias) {
#pragma unroll
        for (int i = 0; i < kTM / 2; ++i) bias_at[lane * (kTM / 2) + i] = bias.of[i];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (p.dtype == MPQ_F16) write_packed<true, kTM, kTN, _Float16>(p, turn, bias_at, c0, t0, lane, acc, between);
        else write_packed<true, kTM, kTN, __bf16>(p, turn, bias_at, c0, t0, lane, acc, between);
    } else {
        if (p.dtype == MPQ_F16) write_packed<false, kTM, kTN, _Float16>(p, turn, bias_at, c0, t0, lane, acc, between);
        else write_packed<false, kTM, kTN, __bf16>(p, turn, bias_at, c0, t0, lane, acc, between);
    }
}

// The tile of this workgroup.  Workgroups are dealt to the eight XCDs in turn,
// and each XCD has an L2 of its own: an XCD takes a run of consecutive tiles, in
// an order that goes through four rows of tiles (of W) side by side, so that the
// 32 workgroups which run there together read 4 + 8 tiles' rows.
constexpr int kXcds = 8, kSide = 4;

// Tile `at` of that order.
__device__ __forceinline__ void tile_at(int at, int tiles_m, int tiles_n, int &tm, int &tn)
{
    const int group = at / (kSide * tiles_n), in = at - group * (kSide * tiles_n);
    const int side = min(kSide, tiles_m - group * kSide);
    tn = __builtin_amdgcn_readfirstlane(in / side);
    tm = __builtin_amdgcn_readfirstlane(group * kSide + in % side);
}

__device__ __forceinline__ bool tile_of(int tiles_m, int tiles_n, int &tm, int &tn)
{
    const int tiles = tiles_m * tiles_n;
    const int xcd = blockIdx.x % kXcds, slot = blockIdx.x / kXcds;
    const int run = tiles / kXcds, more = tiles % kXcds;
    if (slot >= run + (xcd < more ? 1 : 0)) return false;   // the grid is rounded up
    tile_at(xcd * run + min(xcd, more) + slot, tiles_m, tiles_n, tm, tn);
    return true;
}

// Where the tokens of a tile are: rows t0 .. of X behind each other (kGather
// false), or those that a list names, token t0 + i row `list[t0 + i]`.  Offsets into
// all of X's codes, `rows` rows of them, stay below kOutside.
struct MxGather {
    const int32_t *list;
    int64_t rows;
};

// The workgroup of rows c0 .. of W and tokens t0 .. (up to p.n).
template <int kTM, int kTN, bool kGather>
__device__ __forceinline__ void tile_product(const MxProduct &p, int64_t c0, int64_t t0, const MxGather &gather)
{
    constexpr int kBM = 64 * kTM, kBN = 64 * kTN, kRows = kBM + kBN;
    constexpr int kLoads = kRows / 64;                 // of a wavefront a stage
    constexpr int kScaleRows = (kRows + 255) / 256;    // rows whose scales a thread moves
    constexpr int kHalf = 256 * kScaleRows;            // half-words of a stage's scales for one h
    // buffers of their own, which the compiler can tell apart: a read of one
    // does not wait for the loads into another
    __shared__ __align__(16) uint8_t lds0[kRows * kStageBytes], lds1[kRows * kStageBytes];
    __shared__ __align__(16) uint8_t lds2[kRows * kStageBytes], lds3[kRows * kStageBytes];
    __shared__ __align__(16) uint8_t lds_scales[2][4][4 * kHalf];   // of four stages, twice
    const auto ring = [&](int i) { return i == 0 ? lds0 : i == 1 ? lds1 : i == 2 ? lds2 : lds3; };
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane % 32, h = lane / 32;
    const int row_bytes = p.nb * 16;
    const int64_t wrows = min((int64_t)kBM, p.c - c0), xrows = min((int64_t)kBN, p.n - t0);
    const __amdgpu_buffer_rsrc_t wc = buffer_of(p.wc + c0 * row_bytes, wrows * row_bytes);
    const __amdgpu_buffer_rsrc_t xc = kGather ? buffer_of(p.xc, gather.rows * row_bytes)
                                              : buffer_of(p.xc + t0 * row_bytes, xrows * row_bytes);
    const int wm = wave % 2 * (kBM / 2), wn = wave / 2 * (kBN / 2);   // the wavefront's quarter

    // a load covers 16 rows, lane l row l / 4 of them; a wavefront loads a quarter
    // of W's rows (loads 0 .. kTM - 1) and of the tokens'
    const int wrow0 = 16 * wave * kTM, xrow0 = 16 * wave * kTN;
    const uint32_t w_at = tile_lane_offset(wrow0, lane, row_bytes), x_at = tile_lane_offset(xrow0, lane, row_bytes);
    uint32_t gathered[kTN];
    if constexpr (kGather) {
#pragma unroll
        for (int k = 0; k < kTN; ++k) {
            const int at = xrow0 + 16 * k + lane / 4;
            gathered[k] = tile_gather_offset(at < xrows ? gather.list[t0 + at] : -1, lane, row_bytes);
        }
    }
    const auto load = [&](int st, int buf, int k) {
        if (k < kTM)
            load_to_lds(wc, ring(buf) + (wrow0 + 16 * k) * kStageBytes, w_at + tile_stage_offset(k, row_bytes, st, p.nb));
        else if constexpr (kGather)
            load_to_lds(xc, ring(buf) + (kBM + xrow0 + 16 * (k - kTM)) * kStageBytes,
                        tile_gather_stage(gathered[k - kTM], st, p.nb));
        else
            load_to_lds(xc, ring(buf) + (kBM + xrow0 + 16 * (k - kTM)) * kStageBytes,
                        x_at + tile_stage_offset(k - kTM, row_bytes, st, p.nb));
    };
    // scales: a thread moves those of the rows threadIdx.x + 256 i (W's, then the
    // tokens'; a wavefront's 64 are of one kind)
    const auto scales_of = [&](int i) {
        const int row = 256 * i + 64 * wave;
        // (none of them inside the matrix: a buffer of no bytes)
        return row < kBM ? buffer_of(p.ws + (c0 + row) * p.nb, max((int64_t)0, wrows - row) * p.nb)
               : kGather ? buffer_of(p.xs, gather.rows * p.nb)
                         : buffer_of(p.xs + (t0 + row - kBM) * p.nb, max((int64_t)0, xrows - (row - kBM)) * p.nb);
    };
    uint32_t scale_at[kScaleRows];
#pragma unroll
    for (int i = 0; i < kScaleRows; ++i) {
        scale_at[i] = (uint32_t)(lane * p.nb);
        const int row = 256 * i + 64 * wave;
        if (kGather && row >= kBM) {
            const int64_t at = row - kBM + lane, from = at < xrows ? gather.list[t0 + at] : -1;
            scale_at[i] = from < 0 ? kOutside : (uint32_t)(from * p.nb);
        }
    }
    const __amdgpu_buffer_rsrc_t scales0 = scales_of(0), scales1 = scales_of(kScaleRows - 1);
    u32x4 moved[kScaleRows];
    const auto fetch_scales = [&](int four) {   // of the stages 4 four ..
#pragma unroll
        for (int i = 0; i < kScaleRows; ++i)
            moved[i] = load_scales(i == 0 ? scales0 : scales1, scale_at[i] + (uint32_t)(16 * four));
    };
    // row R of W is row R % 32 of tile R / 32 % kTM of its half; rows past kRows
    // are written behind the others and not read
    uint32_t scales_at[kScaleRows];
#pragma unroll
    for (int i = 0; i < kScaleRows; ++i) {
        const int row = (int)threadIdx.x + 256 * i, token = row - kBM;
        scales_at[i] = 2 * (row < kBM   ? row / (32 * kTM) * (32 * kTM) + row % 32 * kTM + row / 32 % kTM
                            : row < kRows ? kBM + token / (32 * kTN) * (32 * kTN) + token % 32 * kTN + token / 32 % kTN
                                          : row);
    }
    const auto place_scales = [&](int four, int w) {   // word w: stage 4 four + w
#pragma unroll
        for (int i = 0; i < kScaleRows; ++i) {
            const uint32_t v = 16 * four + 4 * w < p.nb ? moved[i][w] : 0u;   // past the row: the next row's
            *(half_word *)&lds_scales[four % 2][w][scales_at[i]] = (uint16_t)v;
            *(half_word *)&lds_scales[four % 2][w][2 * kHalf + scales_at[i]] = (uint16_t)(v >> 16);
        }
    };

    f32x16 acc[kTM][kTN];
#pragma unroll
    for (int i = 0; i < kTM; ++i)
#pragma unroll
        for (int j = 0; j < kTN; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;

    fetch_scales(0);
    pin();
#pragma unroll
    for (int st = 0; st < 3; ++st)
#pragma unroll
        for (int k = 0; k < kLoads; ++k) load(st, st, k);
    pin();
#pragma unroll
    for (int w = 0; w < 4; ++w) place_scales(0, w);
    fetch_scales(1);
    Operands<kTM, kTN> first, second;   // of a stage's two steps
    Scales<kTM, kTN> now, next;
    meet<2 * kLoads + kScaleRows>();   // stage 0 is there
#pragma unroll
    for (int i = 0; i < kTM; ++i) first.read(i, ring(0), 0, wm, wn, r, h);
    now.read(lds_scales[0][0], wm, wn, r, h);
    const int fours = (p.nb + 15) / 16;
    for (int four = 0; four < fours; ++four) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int st = 4 * four + q;
            // stage st + 1 is there, and stage st - 1's buffer free; stage st + 2's
            // loads and, where they are as young, the scales' may still run
            if (q == 3 || q == 0) meet<kLoads + kScaleRows>();
            else meet<kLoads>();
            next.read(lds_scales[q == 3 ? (four + 1) % 2 : four % 2][(q + 1) % 4], wm, wn, r, h);
            __builtin_amdgcn_sched_barrier(0);
            // everything else goes out between the products, behind those of
            // each row tile
            multiply_operands<0>(first, now, acc, [&](int i) {
                second.read(i, ring(q), 1, wm, wn, r, h);
                if (i < kLoads) load(st + 3, (q + 3) % 4, i);
                if (q == 2) {
#pragma unroll
                    for (int w = 4 * i / kTM; w < 4 * (i + 1) / kTM; ++w) place_scales(four + 1, w);
                }
            });
            multiply_operands<1>(second, now, acc, [&](int i) {
                first.read(i, ring((q + 1) % 4), 0, wm, wn, r, h);
                if (kTM + i < kLoads) load(st + 3, (q + 3) % 4, kTM + i);
            });
            if (q == 2) {
                pin();
                fetch_scales(four + 2);
                pin();
            }
            now = next;
        }
    }
    // no load into LDS outlives the loop, and no wavefront still reads it
    meet<0>();
    static_assert(kTM % 2 == 0 && 32 * (kTN < 2 ? 1 : 2) * kTurnRow * 4 <= kRows * kStageBytes,
                  "a wavefront's part fits its buffer");
    if constexpr (kGather) {
        static_assert(32 * kTurnRow * 4 + 128 * kTM <= kRows * kStageBytes, "and the bias behind it");
        write_sums<kTM, kTN>(p, ring(wave), (float *)(ring(wave) + 32 * kTurnRow * 4), loaded_bias<kTM>(p, c0 + wm, lane),
                             c0 + wm, t0 + wn, lane, acc, [](int) {});
    } else {
        write_tiles(p, (float *)ring(wave), c0 + wm, t0 + wn, lane, acc);
    }
}

}  // namespace

}  // namespace mpq
