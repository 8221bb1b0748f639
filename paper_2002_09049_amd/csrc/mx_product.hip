// Product of fp4 rows, Y = X W^T + b (mpq_mx_product, mpq_mx_linear), on the
// matrix cores' scaled 4-bit instruction: v_mfma_scale_f32_16x16x128 takes,
// from lane l, the 32 elements of one block of row l % 16 (16 bytes) and that
// block's scale byte, so a block's scale costs nothing beside its product,
// and sums 128 products (four blocks, one for each l / 16) in fp32.  Rows of
// W are the instruction's rows, tokens its columns.
//
// The order of the sum is free as long as both operands share it.
#include <algorithm>
#include <cmath>
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

// The sums of a workgroup's wavefronts to Y.
template <int kNT>
__device__ __forceinline__ void join_waves(const MxProduct &p, float (&part)[kFewWaves][kNT][kWave * 4],
                                           const f32x4 (&acc)[kNT], int64_t c0, int64_t t0)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
#pragma unroll
    for (int t = 0; t < kNT; ++t) *(f32x4 *)&part[wave][t][lane * 4] = acc[t];
    __syncthreads();
    // output o of the tile: row o % 16 of W, token o / 16; lane l's register i
    // holds row 4 (l / 16) + i, token l % 16
    for (int o = threadIdx.x; o < kNT * 256; o += kFewWaves * kWave) {
        const int row = o % 16, tok = o / 16;
        const int at = ((row / 4) * 16 + tok % 16) * 4 + row % 4;
        if (c0 + row >= p.c || t0 + tok >= p.n) continue;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) v += part[w][tok / 16][at];
        if (p.bias) v += p.bias[c0 + row];
        store_y(p.Y, p.dtype, (t0 + tok) * p.ldy + c0 + row, v);
    }
}

template <int kNT>
__global__ void __launch_bounds__(kFewWaves *kWave) mx_few_kernel(MxProduct p)
{
    __shared__ __align__(16) float part[kFewWaves][kNT][kWave * 4];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane % 16, g = lane / 16;
    const int64_t c0 = block_of(blockIdx.z) * 16, t0 = (int64_t)blockIdx.y * 16 * kNT;
    if (c0 >= p.c) return;
    const int nb = p.nb;
    // rows past the end repeat the last one: their sums are not stored
    const int64_t wrow = min(c0 + r, p.c - 1);
    int64_t xrow[kNT];
    f32x4 acc[kNT];
#pragma unroll
    for (int t = 0; t < kNT; ++t) {
        xrow[t] = min(t0 + 16 * t + r, p.n - 1);
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
    int k = wave * kChunkBlocks;
    for (; k + kChunkBlocks <= nb; k += kFewWaves * kChunkBlocks) chunk(std::true_type(), k);
    if (k < nb) chunk(std::false_type(), k);   // the chunk that the row ends in
    join_waves<kNT>(p, part, acc, c0, t0);
}

// One to kN tokens, quantized on the way: a wavefront quantizes its chunk of
// every token itself (eight elements a lane, a block a quad, as
// mx_quantize.hip), through a part of LDS of its own, so the call is one
// launch and X is read by each workgroup.  4096 x 4096, one token: 4.0 us,
// against 1.9 + 3.8 in two launches (and their gap); four tokens, 25088 x 4096:
// 14 us, 3.9 TB/s of W.  With more than four tokens the quantization in every
// workgroup costs more than the launch.
template <int kN, class T>
__global__ void __launch_bounds__(kFewWaves *kWave) mx_token_kernel(MxProduct p, const T *X, int64_t x_ld, int d)
{
    __shared__ __align__(16) float part[kFewWaves][1][kWave * 4];
    __shared__ __align__(16) uint32_t xcodes[kFewWaves][kN][kWave];   // a chunk's codes, eight elements a word
    __shared__ __align__(4) uint8_t xscales[kFewWaves][kN][kChunkBlocks];          // block 4i + g at 4g + i
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane % 16, g = lane / 16;
    const int64_t c0 = block_of(blockIdx.z) * 16;
    if (c0 >= p.c) return;
    const int nb = p.nb;
    const int64_t wrow = min(c0 + r, p.c - 1);
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
        for (int t = 0; t < kN; ++t) c.x[t] = load_eight(X + (t < p.n ? t : 0) * x_ld + e, kWhole ? 8 : d - e);
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
        const bool live = r < kN && r < p.n;
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
    constexpr int kTurn = kFewWaves * kChunkBlocks;
    const int inside = d / kMxBlock;   // whole blocks
    int k = wave * kChunkBlocks;
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
    join_waves<1>(p, part, acc, c0, 0);
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

// The products of one step; after(i) runs behind those of row tile i.
template <int kS, int kTM, int kTN, class After>
__device__ __forceinline__ void multiply_operands(const Operands<kTM, kTN> &o, const Scales<kTM, kTN> &sc,
                                                  f32x16 (&acc)[kTM][kTN], After after)
{
#pragma unroll
    for (int i = 0; i < kTM; ++i) {
#pragma unroll
        for (int j = 0; j < kTN; ++j) {
            // byte of the word: the odd tile's pair is its upper half
            if (i % 2 == 0 && j % 2 == 0)
                acc[i][j] = multiply_tile<kS, kS>(o.a[i], sc.a[i / 2], o.b[j], sc.b[j / 2], acc[i][j]);
            else if (i % 2 == 0)
                acc[i][j] = multiply_tile<kS, kS + 2>(o.a[i], sc.a[i / 2], o.b[j], sc.b[j / 2], acc[i][j]);
            else if (j % 2 == 0)
                acc[i][j] = multiply_tile<kS + 2, kS>(o.a[i], sc.a[i / 2], o.b[j], sc.b[j / 2], acc[i][j]);
            else
                acc[i][j] = multiply_tile<kS + 2, kS + 2>(o.a[i], sc.a[i / 2], o.b[j], sc.b[j / 2], acc[i][j]);
        }
        __builtin_amdgcn_sched_barrier(0);
        after(i);
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

template <int kTM, int kTN>
__device__ __forceinline__ void write_tiles(const MxProduct &p, float *turn, int64_t c0, int64_t t0, int lane,
                                            const f32x16 (&acc)[kTM][kTN])
{
    constexpr int kJ = kTN < 2 ? 1 : 2;   // token tiles of a turn
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

// The tile of this workgroup.  Workgroups are dealt to the eight XCDs in turn,
// and each XCD has an L2 of its own: an XCD takes a run of consecutive tiles, in
// an order that goes through four rows of tiles (of W) side by side, so that the
// 32 workgroups which run there together read 4 + 8 tiles' rows.
constexpr int kXcds = 8, kSide = 4;

__device__ __forceinline__ bool tile_of(int tiles_m, int tiles_n, int &tm, int &tn)
{
    const int tiles = tiles_m * tiles_n;
    const int xcd = blockIdx.x % kXcds, slot = blockIdx.x / kXcds;
    const int run = tiles / kXcds, more = tiles % kXcds;
    if (slot >= run + (xcd < more ? 1 : 0)) return false;   // the grid is rounded up
    const int at = xcd * run + min(xcd, more) + slot;
    const int group = at / (kSide * tiles_n), in = at - group * (kSide * tiles_n);
    const int side = min(kSide, tiles_m - group * kSide);
    tn = __builtin_amdgcn_readfirstlane(in / side);
    tm = __builtin_amdgcn_readfirstlane(group * kSide + in % side);
    return true;
}

template <int kTM, int kTN>
__global__ void __launch_bounds__(256) mx_tile_kernel(MxProduct p)
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
    int tm, tn;
    if (!tile_of((int)((p.c + kBM - 1) / kBM), (int)((p.n + kBN - 1) / kBN), tm, tn)) return;
    const int64_t c0 = (int64_t)tm * kBM, t0 = (int64_t)tn * kBN;
    const int row_bytes = p.nb * 16;
    const int64_t wrows = min((int64_t)kBM, p.c - c0), xrows = min((int64_t)kBN, p.n - t0);
    const __amdgpu_buffer_rsrc_t wc = buffer_of(p.wc + c0 * row_bytes, wrows * row_bytes);
    const __amdgpu_buffer_rsrc_t xc = buffer_of(p.xc + t0 * row_bytes, xrows * row_bytes);
    const int wm = wave % 2 * (kBM / 2), wn = wave / 2 * (kBN / 2);   // the wavefront's quarter

    // a load covers 16 rows, lane l row l / 4 of them; a wavefront loads a quarter
    // of W's rows (loads 0 .. kTM - 1) and of the tokens'
    const int wrow0 = 16 * wave * kTM, xrow0 = 16 * wave * kTN;
    const uint32_t w_at = tile_lane_offset(wrow0, lane, row_bytes), x_at = tile_lane_offset(xrow0, lane, row_bytes);
    const auto load = [&](int st, int buf, int k) {
        if (k < kTM)
            load_to_lds(wc, ring(buf) + (wrow0 + 16 * k) * kStageBytes, w_at + tile_stage_offset(k, row_bytes, st, p.nb));
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
                         : buffer_of(p.xs + (t0 + row - kBM) * p.nb, max((int64_t)0, xrows - (row - kBM)) * p.nb);
    };
    const __amdgpu_buffer_rsrc_t scales0 = scales_of(0), scales1 = scales_of(kScaleRows - 1);
    u32x4 moved[kScaleRows];
    const auto fetch_scales = [&](int four) {   // of the stages 4 four ..
#pragma unroll
        for (int i = 0; i < kScaleRows; ++i)
            moved[i] = load_scales(i == 0 ? scales0 : scales1, (uint32_t)(lane * p.nb + 16 * four));
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
    write_tiles(p, (float *)ring(wave), c0 + wm, t0 + wn, lane, acc);
}

// Some tens of tokens: a workgroup owns 16 rows of W by 64 tokens, 16 for each of
// its four wavefronts, which share W's rows and sum over all of K.  K runs in
// stages of 512 elements, 256 bytes of every row, in a ring as above.  Lanes
// that load for registers directly (mx_few_kernel) are served one by one by
// the vector cache; here 16 lanes load a row's 256 bytes.  Piece q of row r lies in
// place q ^ (r % 16), so the 16 rows that an instruction takes one piece of lie
// in all the banks.  Scales come a ring ahead, a row's 16 bytes a lane
// (wavefront 0: W's, 1: the tokens'), and go to LDS with their words and bytes
// exchanged, as Share has them.
//
// A stage takes 0.3 us, of few workgroups too; a ring of six stages gained
// nothing (64 tokens, 4096 x 4096: 7.0 us, four 5.5, mx_few_kernel 8.3; 25088 x
// 4096: 22.0, 20.7, 34.4; the last is 2.6 TB/s of W).
constexpr int kSlabM = 16, kSlabN = 64, kSlabRows = kSlabM + kSlabN;

// Byte i of word g of the result is byte g of word i.
__device__ __forceinline__ u32x4 transpose_words(u32x4 w)
{
    const uint32_t lo0 = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), lo1 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);
    const uint32_t hi0 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u), hi1 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
    return u32x4{__builtin_amdgcn_perm(lo1, lo0, 0x05040100u), __builtin_amdgcn_perm(lo1, lo0, 0x07060302u),
                 __builtin_amdgcn_perm(hi1, hi0, 0x05040100u), __builtin_amdgcn_perm(hi1, hi0, 0x07060302u)};
}

__global__ void __launch_bounds__(256) mx_slab_kernel(MxProduct p)
{
    constexpr int kLoads = kSlabRows / 16;   // of a wavefront a stage
    __shared__ __align__(16) uint8_t lds0[kSlabRows * kSlabBytes], lds1[kSlabRows * kSlabBytes];
    __shared__ __align__(16) uint8_t lds2[kSlabRows * kSlabBytes], lds3[kSlabRows * kSlabBytes];
    __shared__ __align__(16) uint32_t lds_scales[2][2][kWave][4];   // W's (16 rows), the tokens'
    const auto ring = [&](int i) { return i == 0 ? lds0 : i == 1 ? lds1 : i == 2 ? lds2 : lds3; };
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane % 16, g = lane / 16;
    const int64_t c0 = (int64_t)blockIdx.x * kSlabM, t0 = (int64_t)blockIdx.y * kSlabN;
    const int nb = p.nb, row_bytes = nb * 16;
    const int64_t wrows = min((int64_t)kSlabM, p.c - c0), xrows = min((int64_t)kSlabN, p.n - t0);
    const __amdgpu_buffer_rsrc_t wc = buffer_of(p.wc + c0 * row_bytes, wrows * row_bytes);
    const __amdgpu_buffer_rsrc_t xc = buffer_of(p.xc + t0 * row_bytes, xrows * row_bytes);
    const __amdgpu_buffer_rsrc_t sc = wave == 0 ? buffer_of(p.ws + c0 * nb, wrows * nb)
                                                : buffer_of(p.xs + t0 * nb, wave == 1 ? xrows * nb : 0);
    // a load covers four rows, 4 wave .. of 16: lane l's 16 bytes land in place r of
    // row 4 wave + g
    const auto load = [&](int st, int buf) {
        const uint32_t at = slab_lane_offset(4 * wave + g, r, row_bytes, st, nb);
        load_to_lds(wc, ring(buf) + 4 * wave * kSlabBytes, at);
#pragma unroll
        for (int k = 1; k < kLoads; ++k)
            load_to_lds(xc, ring(buf) + (16 * k + 4 * wave) * kSlabBytes, at + (uint32_t)((k - 1) * 16 * row_bytes));
    };
    u32x4 moved[4];
    const auto fetch_scales = [&](int st, int i) { moved[i] = load_scales(sc, (uint32_t)(lane * nb + 16 * st)); };
    const auto place_scales = [&](int st, int i) {
        u32x4 v = moved[i];
#pragma unroll
        for (int w = 0; w < 4; ++w) v[w] = 16 * st + 4 * w < nb ? v[w] : 0u;   // past the row: the next row's
        if (wave < 2) *(u32x4 *)&lds_scales[i % 2][wave][lane][0] = transpose_words(v);
    };

    f32x4 acc = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int st = -1; st < 3; ++st) {
        fetch_scales(st + 1, st + 1);
        pin();
        if (st >= 0) load(st, st);
        pin();
    }
    place_scales(0, 0);
    const int fours = (nb + 63) / 64;
    for (int four = 0; four < fours; ++four) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int st = 4 * four + q;
            // stage st is there, and stage st - 1's buffer free; the loads of two
            // stages may still run
            meet<2 * (kLoads + 1)>();
            Share a, b;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = ((4 * i + g) ^ r) * 16;
                a.c[i] = *(const u32x4 *)(ring(q) + r * kSlabBytes + at);
                b.c[i] = *(const u32x4 *)(ring(q) + (kSlabM + 16 * wave + r) * kSlabBytes + at);
            }
            a.s = lds_scales[q % 2][0][r][g];
            b.s = lds_scales[q % 2][1][16 * wave + r][g];
            __builtin_amdgcn_sched_barrier(0);
            place_scales(st + 1, (q + 1) % 4);
            fetch_scales(st + 4, q);
            pin();
            load(st + 3, (q + 3) % 4);
            pin();
            acc = multiply_chunk(a, b, acc);
        }
    }
    meet<0>();   // no load into LDS outlives the loop
    const int64_t token = t0 + 16 * wave + r;
    if (token >= p.n) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t row = c0 + 4 * g + i;
        if (row < p.c) store_y(p.Y, p.dtype, token * p.ldy + row, acc[i] + (p.bias ? p.bias[row] : 0.0f));
    }
}

template <int kTM, int kTN>
hipError_t launch_tiles(const MxProduct &p, hipStream_t s)
{
    const int64_t tiles = ((p.c + 64 * kTM - 1) / (64 * kTM)) * ((p.n + 64 * kTN - 1) / (64 * kTN));
    if (!launchable(tiles + kXcds - 1, 256)) return hipErrorInvalidValue;   // more than 2^37 outputs
    LaunchTimer timer(s, kTM == 2 ? (kTN == 1 ? "mx_tile_kernel<2,1>" : "mx_tile_kernel<2,2>")
                                  : (kTN == 2 ? "mx_tile_kernel<4,2>" : "mx_tile_kernel<4,4>"));
    hipLaunchKernelGGL((mx_tile_kernel<kTM, kTN>), dim3((unsigned)((tiles + kXcds - 1) / kXcds * kXcds)), dim3(256), 0, s, p);
    return hipGetLastError();
}

template <int kN>
hipError_t launch_token_as(const MxProduct &p, const void *X, int dtype, int64_t x_ld, int d, hipStream_t s)
{
    const int64_t gx = (p.c + 15) / 16;
    const dim3 grid(grid_x(gx), 1, (unsigned)grid_rows(gx)), threads(kFewWaves * kWave);
    if (dtype == MPQ_F32)
        hipLaunchKernelGGL((mx_token_kernel<kN, float>), grid, threads, 0, s, p, (const float *)X, x_ld, d);
    else if (dtype == MPQ_F16)
        hipLaunchKernelGGL((mx_token_kernel<kN, _Float16>), grid, threads, 0, s, p, (const _Float16 *)X, x_ld, d);
    else
        hipLaunchKernelGGL((mx_token_kernel<kN, __bf16>), grid, threads, 0, s, p, (const __bf16 *)X, x_ld, d);
    return hipGetLastError();
}

}  // namespace

bool mx_quantizes_inside(int64_t n) { return n <= 4; }

hipError_t launch_mx_token(const MxProduct &p, const void *X, int dtype, int64_t x_ld, int64_t d, hipStream_t s)
{
    if (p.n <= 0 || p.c <= 0) return hipSuccess;
    if (!mx_quantizes_inside(p.n) || grid_rows((p.c + 15) / 16) > 65535) return hipErrorInvalidValue;
    LaunchTimer timer(s, "mx_token_kernel");
    return p.n == 1 ? launch_token_as<1>(p, X, dtype, x_ld, (int)d, s) : launch_token_as<4>(p, X, dtype, x_ld, (int)d, s);
}

// Which kernel: the one that a model of its time, in us, finds fastest.  With K
// in stages of 128 elements, a tile kernel takes its start and end plus its
// stages, once for every 256 tiles (one CU each); the slab kernel the same, its
// rings of four stages of 512 whole; the kernel for few tokens, for every 256
// of its workgroups, what the vector cache takes to serve every lane of its
// operands' loads by itself.  The constants are fits to measurements; model
// and time, us, all of one run, for 4096 rows of W:
//    n    d        few        slab       128x64     128x128     256x128     256x256
//    1    4096   4.6  3.5    5.6  5.0    9.9  8.6   12.5 10.4   19.4 15.6   28.8 23.4
//    16   4096   4.6  4.4    5.6  5.2    9.9  8.6   12.5 10.4   19.4 15.6   28.8 23.7
//    32   4096   5.8  5.8    5.6  5.3    9.9  8.7   12.5 10.5   19.4 15.8   28.8 23.7
//    64   4096   8.5  8.3    5.6  5.5    9.9  8.8   12.5 10.7   19.4 16.2   28.8 23.9
//    128  4096  15.0 14.1   10.2  9.8    9.9  9.1   12.5 11.0   19.4 16.7   28.8 25.2
//    512  4096  54.0 48.3   38.0 33.7    9.9 10.8   12.5 12.1   19.4 17.3   28.8 25.7
//    1024 4096   106 89.9   74.9 72.1   19.8 19.9   12.5 15.0   19.4 19.1   28.8 26.9
//    2048 4096   210  175    149  142   39.6 36.8   25.0 30.7   19.4 28.3   28.8 33.3
//    4096 4096   418  349    297  282   79.2 69.7   50.0 58.7   38.9 54.6   28.8 43.0
//    8192 4096   834  697    592  563    158  136    100  112   77.8  103   57.7 81.8
//    16   25088 17.9 14.8   20.6 16.6   42.7 44.6   53.5 51.9   88.3 89.0    131  121
//    32   25088 25.3 21.3   20.6 17.1   42.7 47.9   53.5 52.7   88.3 89.6    131  122
//    64   25088 41.8 34.4   20.6 20.7   42.7 51.3   53.5 55.3   88.3 91.0    131  123
//    128  25088 81.6 65.8   40.2 39.4   42.7 51.0   53.5 67.1   88.3 96.6    131  128
//    1024 25088  639  487    314  294   85.4  103   53.5 77.2   88.3 96.3    131  133
//    64   1024   3.6  4.1    4.3  4.4    5.1  4.8    6.5  5.6    9.4  8.0   14.0 10.7
// Up to four tokens always take the kernel for few: its sums have the order of
// mx_token_kernel's, which a linear call runs for them, so that the two calls
// give the same bits.  (One token and four, d = 4096: 16384 rows of W 8.0 and 9.0
// us, by 128x64 tiles 11.1 and 11.1; 32000 rows 13.6 and 15.5, 12.6 and 12.7;
// 128256 rows 47.2 and 53.8, by 256x128 tiles 47.5 and 48.5.)
// Misses seen: 20 tokens through 4096 x 4096 go to the slabs (5.3 us; the first
// kernel 5.0), 1000 through 512 x 512 to the first kernel (4.5; 128x64 tiles 4.2).
// Where every CU is full, the model says up to a third too little of 128x128 tiles
// and larger and a sixth too much of 128x64; the fastest is the one it takes in
// every row above.  It was fitted with 4096 rows of W.
hipError_t launch_mx_product(const MxProduct &p, hipStream_t s)
{
    if (p.n <= 0 || p.c <= 0) return hipSuccess;
    const double stages = p.nb / 4;
    const auto tiles_us = [&](int tm, int tn, double ends, double stage) {
        const double tiles = (double)((p.c + 64 * tm - 1) / (64 * tm)) * (double)((p.n + 64 * tn - 1) / (64 * tn));
        return ceil(tiles / 256.0) * (ends + stage * stages);
    };
    const double t21 = tiles_us(2, 1, 3.5, 0.2), t22 = tiles_us(2, 2, 4.5, 0.25), t42 = tiles_us(4, 2, 6.0, 0.42),
                 t44 = tiles_us(4, 4, 9.0, 0.62);
    const double best = std::min(std::min(t21, t22), std::min(t42, t44));
    const int nt = p.n <= 16 ? 1 : p.n <= 32 ? 2 : 4;
    const int64_t gx = (p.c + 15) / 16, gy = (p.n + 16 * nt - 1) / (16 * nt);
    const double few = 2.0 + ceil((double)gx * (double)gy / 256.0) * (p.nb / 128.0) * (nt == 1 ? 2.6 : nt == 2 ? 3.8 : 6.5);
    const int64_t sx = (p.c + kSlabM - 1) / kSlabM, sy = (p.n + kSlabN - 1) / kSlabN;
    const double slab = 1.0 + ceil((double)sx * (double)sy / 256.0) * (1.9 + 0.34 * 4.0 * ceil(p.nb / 64.0));
    const bool by_model = !mx_quantizes_inside(p.n);
    if (by_model && slab < best && slab < few && launchable(sx, 256) && sy <= 65535) {
        LaunchTimer timer(s, "mx_slab_kernel");
        hipLaunchKernelGGL(mx_slab_kernel, dim3((unsigned)sx, (unsigned)sy), dim3(256), 0, s, p);
        return hipGetLastError();
    }
    if ((by_model && few > best) || gy > 65535) {
        if (best == t44) return launch_tiles<4, 4>(p, s);
        if (best == t42) return launch_tiles<4, 2>(p, s);
        return best == t22 ? launch_tiles<2, 2>(p, s) : launch_tiles<2, 1>(p, s);
    }
    if (grid_rows(gx) > 65535) return hipErrorInvalidValue;
    LaunchTimer timer(s, "mx_few_kernel");
    auto kern = nt == 1 ? mx_few_kernel<1> : nt == 2 ? mx_few_kernel<2> : mx_few_kernel<4>;
    hipLaunchKernelGGL(kern, dim3(grid_x(gx), (unsigned)gy, (unsigned)grid_rows(gx)), dim3(kFewWaves * kWave), 0, s, p);
    return hipGetLastError();
}

}  // namespace mpq
