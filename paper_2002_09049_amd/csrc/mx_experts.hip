// Products of rows grouped by expert (mpq_mx_experts): row p of Y is
// Q(x) W_e^T + b_e, e the expert with offsets[e] <= p < offsets[e + 1] and x the
// row of X that order names.  The bodies of the products are mx_product.hpp's;
// here a workgroup first finds whose rows it has.
//
// How many rows an expert has is known on the device only, so a grid is sized
// for the most pieces that m rows of E experts can be cut into, min(m, m / T +
// E) of T rows, and workgroups past the last piece end at once.
#include <algorithm>

#include "mx_product.hpp"
#include "mx_quantize.hpp"

namespace mpq {

namespace {

// The row of X that row `at` of Y takes; g.p.n, behind the last, if it names none.
__device__ __forceinline__ int64_t row_of(const MxExperts &g, int64_t at)
{
    if (!g.order) return at < g.p.n ? at : g.p.n;
    const int32_t v = g.order[at];
    const int64_t row = (uint32_t)v / (uint32_t)g.choices;
    return v < 0 || row > g.p.n ? g.p.n : row;
}

// Some rows of one expert.
struct Piece {
    int expert, begin, end, unused;
};

// Inclusive prefix maxima or sums (of numbers >= 0) over the workgroup.
template <class Op>
__device__ __forceinline__ uint32_t prefix(uint32_t v, Op op, uint32_t *waves)
{
    v = op(v, dpp_zero<0x111, 0xF>(v));
    v = op(v, dpp_zero<0x112, 0xF>(v));
    v = op(v, dpp_zero<0x114, 0xF>(v));
    v = op(v, dpp_zero<0x118, 0xF>(v));
    v = op(v, dpp_zero<0x142, 0xA>(v));
    v = op(v, dpp_zero<0x143, 0xC>(v));
    const int wave = threadIdx.x / kWave;
    if (threadIdx.x % kWave == kWave - 1) waves[wave] = v;
    __syncthreads();
    for (int i = 0; i < wave; ++i) v = op(v, waves[i]);
    __syncthreads();
    return v;
}

// The pieces of up to `rows` rows of the groups, in order, behind a first entry
// whose `expert` counts them: prefixes over the experts, four a thread, then a
// thread a piece.
constexpr int kEach = 4;
static_assert(kEach * kRowThreads >= MPQ_MX_MAX_EXPERTS, "");

__device__ __forceinline__ void cut_pieces(const MxExperts &g, int rows, Piece *pieces, int most)
{
    __shared__ uint32_t begin[kEach * kRowThreads + 1], first[kEach * kRowThreads + 1], waves[kRowThreads / kWave];
    const int e0 = threadIdx.x * kEach, m = (int)g.m;
    // where the groups end: prefix maxima of the offsets behind the first
    uint32_t end[kEach], top = (uint32_t)min(max(g.offsets[0], 0), m);
    const uint32_t start = top;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (e0 + i < g.experts) top = max(top, (uint32_t)min(max(g.offsets[e0 + i + 1], 0), m));
        end[i] = top;
    }
    const uint32_t upto = prefix(top, MaxOp(), waves);
    begin[e0 + kEach] = upto;
    if (threadIdx.x == 0) begin[0] = start;
    __syncthreads();
    const uint32_t from = begin[e0];
    uint32_t count[kEach], sum = 0, at = from;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        end[i] = max(end[i], from);
        count[i] = (end[i] - at + (uint32_t)rows - 1) / (uint32_t)rows;
        sum += count[i];
        at = end[i];
        if (i + 1 < kEach) begin[e0 + i + 1] = end[i];
    }
    uint32_t before = prefix(sum, SumOp(), waves) - sum;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        first[e0 + i] = before;
        before += count[i];
    }
    if (threadIdx.x == kRowThreads - 1) first[kEach * kRowThreads] = before;
    __syncthreads();
    const int all = min((int)first[kEach * kRowThreads], most);
    if (threadIdx.x == 0) pieces[0] = Piece{all, 0, 0, 0};
    for (int i = threadIdx.x; i < all; i += kRowThreads) {
        const int x = last_at_most(g.experts, i, [&](int j) { return (int)first[j]; });
        const int b = (int)begin[x] + (i - (int)first[x]) * rows;
        pieces[1 + i] = Piece{x, b, min(b + rows, (int)begin[x + 1]), 0};
    }
}

// The pieces, by the first workgroup; the list of X's rows that Y's take, by the
// next `listing`; by the others the rows of X to fp4 blocks, behind them one of
// zeros.
template <class T>
__global__ void __launch_bounds__(kRowThreads) mx_prepare_kernel(MxExperts g, const T *X, int64_t x_ld, int d, int rows,
                                                                 int most, int listing, int32_t *list, uint8_t *codes,
                                                                 uint8_t *scales)
{
    if ((int)blockIdx.x > listing) {
        quantize_eight((int64_t)blockIdx.x - 1 - listing, X, g.p.n, d, x_ld, g.p.nb * kMxBlock, codes, scales);
        return;
    }
    if (blockIdx.x > 0) {
        const int64_t at = (int64_t)(blockIdx.x - 1) * kRowThreads + threadIdx.x;
        if (at < g.m) list[at] = (int32_t)row_of(g, at);
        return;
    }
    const int nb = g.p.nb;
    for (int i = threadIdx.x; i < 4 * nb; i += kRowThreads) ((uint32_t *)(codes + g.p.n * nb * 16))[i] = 0;
    for (int i = threadIdx.x; i < nb / 4; i += kRowThreads) ((uint32_t *)(scales + g.p.n * nb))[i] = 0;
    cut_pieces(g, rows, (Piece *)g.pieces, most);
}

// An entry of the list, which no kernel that reads it writes: by scalar loads.
typedef const int32_t __attribute__((address_space(4))) * constant_ints;
__device__ __forceinline__ Piece piece_at(const Piece *pieces, int i)
{
    const constant_ints from = (constant_ints)(uintptr_t)(pieces + i);
    return Piece{from[0], from[1], from[2], 0};
}

// The product of one expert: its weights and bias, tokens up to `end`.
__device__ __forceinline__ MxProduct product_of(const MxExperts &g, int expert, int end)
{
    MxProduct p = g.p;
    const int64_t rows = (int64_t)expert * p.c;
    p.wc += rows * p.nb * 16;
    p.ws += rows * p.nb;
    if (p.bias) p.bias += rows;
    p.n = end;
    return p;
}

template <int kNT, int kSplit>
__global__ void __launch_bounds__(kFewWaves *kWave) mx_experts_few_kernel(MxExperts g, int row_blocks)
{
    const Piece *pieces = (const Piece *)g.pieces;
    const int i = blockIdx.x / (unsigned)row_blocks;
    if (i >= piece_at(pieces, 0).expert) return;
    const Piece q = piece_at(pieces, 1 + i);
    const int32_t *list = g.list;
    few_product<kNT, kSplit>(product_of(g, q.expert, q.end),
                             (int64_t)(blockIdx.x - (unsigned)i * row_blocks) * kFewRows<kSplit>, q.begin,
                             [=](int64_t at) { return (int64_t)list[at]; });
}

// One to four rows of X: as mx_token_kernel, a workgroup for each run of kN rows
// of a group, started by the run's first row.  Every wavefront finds the group of
// row p from the offsets itself.
template <int kN, int kSplit, class T>
__global__ void __launch_bounds__(kFewWaves *kWave) mx_experts_token_kernel(MxExperts g, const T *X, int64_t x_ld, int d)
{
    const int p = blockIdx.y, lane = threadIdx.x % kWave;
    // the first group that ends behind p, and the largest offset before that end
    int e = -1, end = 0, before = lane == 0 ? g.offsets[0] : 0;
    for (int i = 0; i < g.experts && e < 0; i += kWave) {
        const int at = i + lane < g.experts ? g.offsets[i + lane + 1] : -1;
        const unsigned long long behind = __ballot(at > p);
        const int first = behind ? __builtin_ctzll(behind) : kWave;
        if (lane < first) before = max(before, at);
        if (behind) {
            e = i + first;
            end = readlane(at, first);
        }
    }
    if (e < 0) return;
    const int begin = __builtin_amdgcn_readfirstlane(wave_reduce(before, MaxOp()));
    end = __builtin_amdgcn_readfirstlane(min(end, (int)g.m));
    e = __builtin_amdgcn_readfirstlane(e);
    if (p < begin || (p - begin) % kN != 0) return;
    const int n = min(kN, end - p);
    int64_t row[kN];
#pragma unroll
    for (int t = 0; t < kN; ++t) row[t] = row_of(g, p + min(t, n - 1));
    token_product<kN, kSplit, T>(
        product_of(g, e, p + n), (int64_t)blockIdx.x * kFewRows<kSplit>, p, n, d,
        [&](int t) { return X + (row[t] < g.p.n ? row[t] : 0) * x_ld; }, [&](int t) { return row[t] >= g.p.n; });
}

template <int kTM, int kTN>
__global__ void __launch_bounds__(256) mx_experts_tile_kernel(MxExperts g)
{
    constexpr int kBM = 64 * kTM;
    const Piece *pieces = (const Piece *)g.pieces;
    int tm, i;
    if (!tile_of((int)((g.p.c + kBM - 1) / kBM), piece_at(pieces, 0).expert, tm, i)) return;
    const Piece q = piece_at(pieces, 1 + i);
    tile_product<kTM, kTN, true>(product_of(g, q.expert, q.end), (int64_t)tm * kBM, q.begin,
                                 MxGather{g.list, g.p.n + 1});
}

// Many rows for most experts: tiles of 256 rows of W by 256 tokens, as
// mx_tile_kernel's (mx_product.hpp has the ring), by workgroups that stay, one a CU,
// and take their XCD's tiles in turn.  What a tile is, which rows of X it has and
// its first three stages are each loads that wait for the ones before: done tile
// by tile they took 8 of 25 us at d = 2048.  So the next tile's piece is read, and
// its first stages are loaded, while the sums of this one are written, whose way
// through LDS takes the ring's fourth buffer, and the rows of the one after while
// this one is multiplied.  65536 rows for 64 experts, timed in turn with tiles of
// 256 x 256 that do not stay: 5632 x 2048 551 us and 591, 2048 x 2816 285 and 305.
// 43% of the CUs' cycles are products, and the others are what bounds it: at the clock
// that it runs at, 1.8 GHz, products alone would be 7.5 PFLOP/s, and it reaches 2.6 to 3.0.
__global__ void __launch_bounds__(256) mx_experts_stay_kernel(MxExperts g)
{
    constexpr int kTM = 4, kTN = 4, kBM = 64 * kTM, kBN = 64 * kTN, kRows = kBM + kBN;
    constexpr int kLoads = kRows / 64, kHalf = kRows;
    __shared__ __align__(16) uint8_t lds0[kRows * kStageBytes], lds1[kRows * kStageBytes];
    __shared__ __align__(16) uint8_t lds2[kRows * kStageBytes], lds3[kRows * kStageBytes];
    __shared__ __align__(16) uint8_t lds_scales[2][4][4 * kHalf];
    __shared__ __align__(16) float lds_bias[4][32 * kTM];
    const auto ring = [&](int i) { return i == 0 ? lds0 : i == 1 ? lds1 : i == 2 ? lds2 : lds3; };
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r = lane % 32, h = lane / 32;
    const Piece *pieces = (const Piece *)g.pieces;
    const int nb = g.p.nb, row_bytes = nb * 16;
    const int wm = wave % 2 * (kBM / 2), wn = wave / 2 * (kBN / 2);   // the wavefront's quarter
    const int row0 = 16 * wave * kTM;                                 // its loads' rows, of W and of X

    // this XCD's run of tiles, dealt to its workgroups in turn
    const int tiles_m = (int)((g.p.c + kBM - 1) / kBM), tiles_n = piece_at(pieces, 0).expert, tiles = tiles_m * tiles_n;
    const int xcd = blockIdx.x % kXcds, step = gridDim.x / kXcds;
    const int run = tiles / kXcds, more = tiles % kXcds, begin = xcd * run + min(xcd, more);
    const int end = begin + run + (xcd < more ? 1 : 0);
    int at = begin + blockIdx.x / kXcds, tm, tn;
    if (at >= end) return;

    // the tile at hand
    MxProduct p;
    int64_t c0, t0;
    __amdgpu_buffer_rsrc_t wc = buffer_of(g.p.wc, 0), scales_w = wc;
    const __amdgpu_buffer_rsrc_t xc = buffer_of(g.p.xc, (g.p.n + 1) * row_bytes);
    const __amdgpu_buffer_rsrc_t scales_x = buffer_of(g.p.xs, (g.p.n + 1) * nb);
    uint32_t gathered[kTN], scale_at;
    const uint32_t w_at = tile_lane_offset(row0, lane, row_bytes);

    // the lane's entries of the list for a piece: those that its loads begin with
    // (row row0 + 16 k + lane / 4), and its scales' (row 64 wave + lane)
    int32_t codes_of[kTN], scales_of;
    const auto fetch_rows = [&](const Piece &q) {
        const auto entry = [&](int i) { return g.list[min(q.begin + i, q.end - 1)]; };
#pragma unroll
        for (int k = 0; k < kTN; ++k) codes_of[k] = entry(row0 + 16 * k + lane / 4);
        scales_of = entry(64 * wave + lane);
    };
    const auto take = [&](const Piece &q) {   // the tile (tm, piece q) from the entries fetched
        p = product_of(g, q.expert, q.end);
        c0 = (int64_t)tm * kBM;
        t0 = q.begin;
#pragma unroll
        for (int k = 0; k < kTN; ++k) {
            const bool live = row0 + 16 * k + lane / 4 < q.end - q.begin;
            gathered[k] = tile_gather_offset(live ? codes_of[k] : -1, lane, row_bytes);
        }
        scale_at = 64 * wave + lane < q.end - q.begin ? (uint32_t)(scales_of * nb) : kOutside;
        const int64_t wrows = min((int64_t)kBM, p.c - c0);
        wc = buffer_of(p.wc + c0 * row_bytes, wrows * row_bytes);
        scales_w = buffer_of(p.ws + (c0 + 64 * wave) * nb, max((int64_t)0, wrows - 64 * wave) * nb);
    };
    const auto load = [&](int st, int buf, int k) {
        if (k < kTM)
            load_to_lds(wc, ring(buf) + (row0 + 16 * k) * kStageBytes, w_at + tile_stage_offset(k, row_bytes, st, nb));
        else
            load_to_lds(xc, ring(buf) + (kBM + row0 + 16 * (k - kTM)) * kStageBytes,
                        tile_gather_stage(gathered[k - kTM], st, nb));
    };
    u32x4 moved_w, moved_x;
    const auto fetch_scales = [&](int four) {   // of the stages 4 four ..
        moved_w = load_scales(scales_w, (uint32_t)(lane * nb + 16 * four));
        moved_x = load_scales(scales_x, scale_at + (uint32_t)(16 * four));
    };
    // row R of 256 is row R % 32 of tile R / 32 % 4 of its half
    const int thread = threadIdx.x, place = 2 * (thread / 128 * 128 + thread % 32 * 4 + thread / 32 % 4);
    const auto place_scales = [&](int four, int w) {   // word w: stage 4 four + w
        const bool live = 16 * four + 4 * w < nb;      // past the row: the next row's
        const uint32_t vw = live ? moved_w[w] : 0u, vx = live ? moved_x[w] : 0u;
        uint8_t *to = lds_scales[four % 2][w] + place;
        *(half_word *)to = (uint16_t)vw;
        *(half_word *)(to + 2 * kHalf) = (uint16_t)(vw >> 16);
        *(half_word *)(to + 2 * kBM) = (uint16_t)vx;
        *(half_word *)(to + 2 * kBM + 2 * kHalf) = (uint16_t)(vx >> 16);
    };
    const auto stage = [&](int st) {   // one of a tile's first three, each to its buffer
        pin();
#pragma unroll
        for (int k = 0; k < kLoads; ++k) load(st, st, k);
        pin();
    };
    const auto begin_tile = [&]() {   // its scales' first loads, then the first stage
        pin();
        fetch_scales(0);
        stage(0);
    };

    tile_at(at, tiles_m, tiles_n, tm, tn);
    Piece next = piece_at(pieces, 1 + tn);
    fetch_rows(next);
    take(next);
    begin_tile();
    stage(1);
    stage(2);
    at += step;
    if (at < end) {
        tile_at(at, tiles_m, tiles_n, tm, tn);
        next = piece_at(pieces, 1 + tn);
    }
    const int fours = (nb + 15) / 16;
    for (;;) {
        if (at < end) fetch_rows(next);
        f32x16 acc[kTM][kTN];
#pragma unroll
        for (int i = 0; i < kTM; ++i)
#pragma unroll
            for (int j = 0; j < kTN; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) place_scales(0, w);
        pin();
        fetch_scales(1);
        Operands<kTM, kTN> first, second;   // of a stage's two steps
        Scales<kTM, kTN> now, then;
        meet<2 * kLoads + 2>();   // stage 0 is there
#pragma unroll
        for (int i = 0; i < kTM; ++i) first.read(i, ring(0), 0, wm, wn, r, h);
        now.read(lds_scales[0][0], wm, wn, r, h);
        for (int four = 0; four < fours; ++four) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int st = 4 * four + q;
                // stage st + 1 is there, and stage st - 1's buffer free; stage st +
                // 2's loads and, where they are as young, the scales' may still run
                if (q == 3 || q == 0) meet<kLoads + 2>();
                else meet<kLoads>();
                then.read(lds_scales[q == 3 ? (four + 1) % 2 : four % 2][(q + 1) % 4], wm, wn, r, h);
                __builtin_amdgcn_sched_barrier(0);
                multiply_spread<0>(first, now, acc, [&](int i, int j) {
                    if (j == 0) second.read_one<false>(i, ring(q), 1, wm, wn, r, h);
                    if (j == 1) second.read_one<true>(i, ring(q), 1, wm, wn, r, h);
                    if (j == 2) load(st + 3, (q + 3) % 4, i);
                    if (j == 3 && q == 2) place_scales(four + 1, i);
                });
                multiply_spread<1>(second, now, acc, [&](int i, int j) {
                    if (j == 0) first.read_one<false>(i, ring((q + 1) % 4), 0, wm, wn, r, h);
                    if (j == 1) first.read_one<true>(i, ring((q + 1) % 4), 0, wm, wn, r, h);
                    if (j == 2) load(st + 3, (q + 3) % 4, kTM + i);
                });
                if (q == 2) {
                    pin();
                    fetch_scales(four + 2);
                    pin();
                }
                now = then;
            }
        }
        // no load into LDS outlives the loop, and no wavefront still reads it
        meet<0>();
        const MxProduct done = p;
        const int64_t done_c0 = c0, done_t0 = t0;
        const bool last = at >= end;
        // (before the ring's next loads, not to wait for those)
        const Bias<kTM> bias = loaded_bias<kTM>(done, done_c0 + wm, lane);
        if (!last) {
            take(next);
            begin_tile();
            at += step;
            if (at < end) {
                tile_at(at, tiles_m, tiles_n, tm, tn);
                next = piece_at(pieces, 1 + tn);
            }
        }
        static_assert(32 * kTurnRow * 4 * 4 <= kRows * kStageBytes, "the four wavefronts' parts fit the buffer");
        write_sums<kTM, kTN>(done, lds3 + wave * (32 * kTurnRow * 4), lds_bias[wave], bias, done_c0 + wm, done_t0 + wn, lane,
                             acc, [&](int j) {
                                 if (j < 2 && !last) stage(j + 1);
                             });
        if (last) return;
    }
}

template <int kNT, int kSplit>
hipError_t launch_few(const MxExperts &g, int64_t pieces, hipStream_t s)
{
    const int64_t gx = (g.p.c + kFewRows<kSplit> - 1) / kFewRows<kSplit>;
    LaunchTimer timer(s, "mx_experts_few_kernel");
    hipLaunchKernelGGL((mx_experts_few_kernel<kNT, kSplit>), dim3((unsigned)(gx * pieces)), dim3(kFewWaves * kWave), 0, s, g,
                       (int)gx);
    return hipGetLastError();
}

template <int kTM, int kTN>
hipError_t launch_tiles(const MxExperts &g, int64_t pieces, hipStream_t s)
{
    const int64_t tiles = (g.p.c + 64 * kTM - 1) / (64 * kTM) * pieces;
    LaunchTimer timer(s, kTN == 1 ? "mx_experts_tile_kernel<2,1>" : "mx_experts_tile_kernel<2,2>");
    hipLaunchKernelGGL((mx_experts_tile_kernel<kTM, kTN>), dim3((unsigned)((tiles + kXcds - 1) / kXcds * kXcds)), dim3(256),
                       0, s, g);
    return hipGetLastError();
}

template <int kSplit, class T>
hipError_t launch_token_split(const MxExperts &g, const T *X, int64_t x_ld, int d, hipStream_t s)
{
    const dim3 grid((unsigned)((g.p.c + kFewRows<kSplit> - 1) / kFewRows<kSplit>), (unsigned)g.m), threads(kFewWaves * kWave);
    if (g.p.n == 1) hipLaunchKernelGGL((mx_experts_token_kernel<1, kSplit, T>), grid, threads, 0, s, g, X, x_ld, d);
    else hipLaunchKernelGGL((mx_experts_token_kernel<4, kSplit, T>), grid, threads, 0, s, g, X, x_ld, d);
    return hipGetLastError();
}

// How many wavefronts share 16 rows of W (by splitting K): as many as leave the
// workgroups, which all run at once then, few enough.  One token, 8 experts, us
// by shares of 1, 2, 4, 8 (workgroups of the one taken: 128, 256, 256, 704):
//   c 256, d 2048    9.3  7.2  6.2  5.8      c 256, d 8192    23.1 13.9  9.5  7.3
//   c 1024, d 2048   9.5  7.3  6.3  7.5      c 1024, d 8192   24.6 15.4 10.6 12.1
//   c 2048, d 2048   9.6  7.4  7.5 11.0      c 2048, d 8192   25.0 17.3 17.5 21.7
//   c 5632, d 2048  15.7 14.6 16.7 26.4      c 5632, d 8192   44.5 35.0 36.1 47.8
// Four tokens (whose rows are quantized by every wavefront): c 256, d 2048 11.5 8.5
// 7.4 9.3; c 1024, d 2048 12.5 14.0 18.0 23.2; c 2048, d 512 10.8 15.9 24.2 34.7.
// (Three of 256 rows of W, 384 workgroups by eight: 8.8, and by four 7.3: there the
// bound that one token's times give is too high.)
template <class T>
hipError_t launch_token(const MxExperts &g, const T *X, int64_t x_ld, int d, hipStream_t s)
{
    const auto groups = [&](int rows) { return (g.p.c + rows - 1) / rows * g.m; };
    if (groups(16) <= 384) return launch_token_split<8>(g, X, x_ld, d, s);
    if (groups(32) <= 384) return launch_token_split<4>(g, X, x_ld, d, s);
    if (groups(64) <= 384 || g.p.n == 1) return launch_token_split<2>(g, X, x_ld, d, s);
    return launch_token_split<1>(g, X, x_ld, d, s);
}

hipError_t launch_stay(const MxExperts &g, int64_t pieces, hipStream_t s)
{
    // (a multiple of kXcds, and of every CU one)
    const int64_t tiles = (g.p.c + 255) / 256 * pieces, blocks = std::min((int64_t)256, (tiles + kXcds - 1) / kXcds * kXcds);
    LaunchTimer timer(s, "mx_experts_stay_kernel");
    hipLaunchKernelGGL(mx_experts_stay_kernel, dim3((unsigned)blocks), dim3(256), 0, s, g);
    return hipGetLastError();
}

template <class T>
hipError_t launch_prepare(const MxExperts &g, const T *X, int64_t x_ld, int d, int rows, int most, int32_t *list,
                          uint8_t *codes, uint8_t *scales, hipStream_t s)
{
    // below 2^22 workgroups: (n + 1) rows of less than 2^32 elements in all, m of at most 2^26
    const int64_t listing = (g.m + kRowThreads - 1) / kRowThreads;
    const int64_t blocks = 1 + listing + (g.p.n * g.p.nb * kMxBlock + kRowElems - 1) / kRowElems;
    hipLaunchKernelGGL(mx_prepare_kernel<T>, dim3((unsigned)blocks), dim3(kRowThreads), 0, s, g, X, x_ld, d, rows, most,
                       (int)listing, list, codes, scales);
    return hipGetLastError();
}

int64_t most_pieces(int64_t m, int64_t experts, int rows) { return std::min(m, m / rows + experts); }

// How a call is done: inside one launch (rows 0), or in pieces of so many rows, by
// wavefronts that load for themselves (few) or by tiles.
struct Way {
    int rows;
    bool few;
};

// By a model of the times, us, as launch_mx_product's: a round of 256 tiles takes
// its ends and its stages of K; of m rows of E experts about E (mean / rows + 1 / 2)
// pieces come, at least E, and half a round is lost at the end.  The launch before
// is not in it, as it is the same for all of them; the times measured have it (4 us
// for few rows, 13 for 8192 of 2048, 17 for 4096 of 8192: of the 61.0 us below, where
// the model gives the tiles 32, they take 48).  us, bf16, 64 experts of 2048 x 2048:
//    mean rows    8    16    32    48    64    100   128   200   256   400   700  1024
//    wavefronts  41.9  55.6  89.4   124   158   236   294   447   566   871  1505  2193
//    128 x 64    33.4  33.0  36.9  39.0  40.6  51.0  56.2  76.9  94.9   137   235   324
//    128 x 128   36.2  35.8  36.9  38.2  42.6  47.8  49.9  68.1  76.1   109   188   265
//    256 x 256   48.5  48.1  49.2  49.9  51.4  69.9  70.6  72.7  75.6   111   162   215
// and 4 experts of 1024 x 8192: mean 64 43.3, 23.6, 25.5, 54.0; 1024 -, 68.0, 61.0, 68.9.
// (256 x 128 tiles were the fastest in one of 30 cases.)  Wavefronts that load for
// themselves win while few rows have most experts to themselves (mean 1.2, 64 of
// 2048 x 2816: 30.7, tiles 33.3; of 2048 x 8192: 71, 93; mean 4.8: 41.1 and 37.3)
// or tiles are too few to fill the CUs (8 experts, mean 4, of 256 x 8192: 11.6,
// 21.3; of 2048 x 2816: 12.0, 13.4).
//
// Up to four tokens go in one launch, unless several read much of W.  64 experts, 8
// choices, us in one launch and in two (each side forced, on the same kernels):
//    c x d         one token    two           three         four
//    1024 x 512    5.6   8.4    6.6   8.9     9.5   9.4     7.0   9.4
//    1024 x 2048   6.3   9.2    8.4  10.9    12.9  13.6    12.2  14.4
//    1024 x 8192  10.5  14.1   19.1  20.6    31.9  24.0    30.5  29.0
//    2048 x 512    5.8   8.6    7.1   9.4    10.3  10.0    10.4  10.5
//    2048 x 2048   7.4  10.6   12.2  14.0    20.0  17.2    20.6  17.3
//    2048 x 8192  17.3  21.0   30.8  29.5    54.2  39.1    56.3  48.7
//    5632 x 512    7.7   9.8   13.5  12.4    17.9  14.3    22.1  16.8
//    5632 x 2048  14.3  17.0   29.2  25.4    37.6  30.8    45.9  36.0
//    5632 x 8192  34.9  40.6   90.4  68.0     130   101     182   131
// (256 rows of W: one launch is the faster throughout.)  40 MB of W leaves three on the
// slower side: 5632 x 512 with two and three tokens (25 and 37 MB: 1.10 and 1.24 of
// the faster one) and 1024 x 8192 with two (71 MB: 1.07).  What the bytes do not
// count is that each of c / 64 times m workgroups quantizes its rows itself.
Way way_of(int64_t n, int64_t m, int64_t experts, int64_t c, int64_t d)
{
    const double weights = (double)m * (double)c * (double)mx_row(d) * 17.0 / 32.0;
    // (the workgroups of the two that load for themselves, of 64 rows where they are
    // many, count their threads in 32 bits; the tiles, which are fewer, are checked by the caller)
    const auto fits = [&](int64_t pieces) { return launchable((c + 63) / 64 * pieces, kFewWaves * kWave); };
    if (mx_quantizes_inside(n) && m <= 64 && (n == 1 || weights <= 40e6) && fits(m)) return Way{0, true};
    const double mean = (double)m / (double)experts, stages = (double)mx_row(d) / 128.0;
    const double pieces = (double)std::min(m, experts);
    if ((mean <= 2.0 || (mean <= 16.0 && pieces * (double)((c + 127) / 128) < 256.0)) && fits(4 * most_pieces(m, experts, 16)))
        return Way{16, true};
    const auto time = [&](int64_t bm, int64_t bn, double ends, double stage) {
        const double tiles = (double)((c + bm - 1) / bm) * (double)experts * std::max(1.0, mean / (double)bn + 0.5);
        return std::max(1.0, tiles / 256.0 + 0.5) * (ends + stage * stages);
    };
    const double t64 = time(128, 64, 3.5, 0.2), t128 = time(128, 128, 4.5, 0.25), t256 = time(256, 256, 11.0, 0.8);
    if (t256 < t64 && t256 < t128) return Way{256, false};
    return Way{t128 < t64 ? 128 : 64, false};
}

// Shares of K among the wavefronts: two chunks of 512 a wavefront, more of them
// where the workgroups would be fewer than CUs (60 experts, mean 4.8, of c x d, by
// shares of 1, 2, 4, 8: 2048 x 512 15.0 15.4 17.3 23.3; 2048 x 2816 43.3 42.0 41.1
// 44.6; 2048 x 8192 135 124 116 115; 8 experts of 256 x 2816 16.1 12.0 10.2 9.2).
hipError_t launch_few_rows(const MxExperts &g, int64_t pieces, hipStream_t s)
{
    const int chunks = (g.p.nb + kChunkBlocks - 1) / kChunkBlocks;
    int split = chunks <= 4 ? 2 : chunks <= 8 ? 4 : 8;
    while (split < 8 && (g.p.c * split + 127) / 128 * std::min(g.m, (int64_t)g.experts) < 256) split *= 2;
    if (split == 2) return launch_few<1, 2>(g, pieces, s);
    return split == 4 ? launch_few<1, 4>(g, pieces, s) : launch_few<1, 8>(g, pieces, s);
}

}  // namespace

// The quantized rows of X and one of zeros, the pieces, and the list of rows.  The
// pieces are counted as the smallest ones, of 16 rows, whatever the way: so what a
// call takes does not fall as n, m, experts, c or d grow.
size_t mx_experts_bytes(int64_t n, int64_t m, int64_t experts, int64_t c, int64_t d)
{
    const Way way = way_of(n, m, experts, c, d);
    if (way.rows == 0) return 0;
    const int64_t w = mx_row(d);
    return (size_t)((n + 1) * (w / 2) + ((n + 1) * (w / 32) + 15) / 16 * 16)
           + sizeof(Piece) * (size_t)(1 + most_pieces(m, experts, 16)) + (size_t)m * sizeof(int32_t);
}

hipError_t launch_mx_experts(MxExperts g, const void *X, int dtype, int64_t x_ld, int64_t d, uint8_t *space, hipStream_t s)
{
    const int64_t n = g.p.n, w = mx_row(d);
    const Way way = way_of(n, g.m, g.experts, g.p.c, d);
    if (way.rows == 0) {
        LaunchTimer timer(s, "mx_experts_token_kernel");
        if (dtype == MPQ_F32) return launch_token(g, (const float *)X, x_ld, (int)d, s);
        if (dtype == MPQ_F16) return launch_token(g, (const _Float16 *)X, x_ld, (int)d, s);
        return launch_token(g, (const __bf16 *)X, x_ld, (int)d, s);
    }
    uint8_t *xc = space, *xs = xc + (n + 1) * (w / 2);
    Piece *pieces = (Piece *)(xs + ((n + 1) * (w / 32) + 15) / 16 * 16);
    g.p.xc = xc;
    g.p.xs = xs;
    g.pieces = pieces;
    const int64_t most = most_pieces(g.m, g.experts, way.rows), of = way.rows == 256 ? 256 : 128;   // rows of W of a tile
    if (!way.few && !launchable((g.p.c + of - 1) / of * most + kXcds - 1, 256)) return hipErrorInvalidValue;
    int32_t *list = (int32_t *)(pieces + 1 + most);
    g.list = list;
    hipError_t e;
    {
        LaunchTimer timer(s, "mx_prepare_kernel");
        e = dtype == MPQ_F32 ? launch_prepare(g, (const float *)X, x_ld, (int)d, way.rows, (int)most, list, xc, xs, s)
            : dtype == MPQ_F16 ? launch_prepare(g, (const _Float16 *)X, x_ld, (int)d, way.rows, (int)most, list, xc, xs, s)
                               : launch_prepare(g, (const __bf16 *)X, x_ld, (int)d, way.rows, (int)most, list, xc, xs, s);
    }
    if (e != hipSuccess) return e;
    if (way.few) return launch_few_rows(g, most, s);
    if (way.rows == 64) return launch_tiles<2, 1>(g, most, s);
    if (way.rows == 128) return launch_tiles<2, 2>(g, most, s);
    return launch_stay(g, most, s);
}

}  // namespace mpq
