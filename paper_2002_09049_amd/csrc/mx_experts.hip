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

namespace mpq {

namespace {

// Some rows of one expert.
struct Piece {
    int expert, begin, end, unused;
};

// The pieces of up to `rows` rows of the groups, in order, behind a first entry
// whose `expert` counts them.  One workgroup: prefixes over at most 1024 experts
// in LDS, then a thread a piece.
constexpr int kPieceThreads = 1024;
__global__ void __launch_bounds__(kPieceThreads) mx_pieces_kernel(const int32_t *offsets, int experts, int m, int rows,
                                                                  Piece *pieces, int most, uint32_t *zeros_codes,
                                                                  uint32_t *zeros_scales, int nb)
{
    __shared__ int begin[kPieceThreads + 1], first[kPieceThreads + 1];
    const int e = threadIdx.x;
    // X's row of zeros
    for (int i = e; i < 4 * nb; i += kPieceThreads) zeros_codes[i] = 0;
    for (int i = e; i < nb / 4; i += kPieceThreads) zeros_scales[i] = 0;
    // begins: prefix maxima
    if (e <= experts) begin[e] = min(max(offsets[e], 0), m);
    if (e == 0 && experts == kPieceThreads) begin[experts] = min(max(offsets[experts], 0), m);
    __syncthreads();
    for (int step = 1; step <= experts; step *= 2) {
        const int a = e <= experts && e >= step ? begin[e - step] : 0;
        const int last = experts == kPieceThreads ? begin[experts - step] : 0;
        __syncthreads();
        if (e <= experts) begin[e] = max(begin[e], a);
        if (e == 0 && experts == kPieceThreads) begin[experts] = max(begin[experts], last);
        __syncthreads();
    }
    if (e < experts) first[e + 1] = (begin[e + 1] - begin[e] + rows - 1) / rows;
    if (e == 0) first[0] = 0;
    __syncthreads();
    for (int step = 1; step < experts; step *= 2) {
        const int a = e < experts && e >= step ? first[e + 1 - step] : 0;
        __syncthreads();
        if (e < experts) first[e + 1] += a;
        __syncthreads();
    }
    const int count = min(first[experts], most);
    if (e == 0) pieces[0] = Piece{count, 0, 0, 0};
    for (int i = e; i < count; i += kPieceThreads) {
        const int x = last_at_most(experts, i, [&](int j) { return first[j]; });
        const int at = begin[x] + (i - first[x]) * rows;
        pieces[1 + i] = Piece{x, at, min(at + rows, begin[x + 1]), 0};
    }
}

__device__ __forceinline__ Piece piece_at(const Piece *pieces, int i)
{
    Piece q = pieces[i];
    q.expert = __builtin_amdgcn_readfirstlane(q.expert);
    q.begin = __builtin_amdgcn_readfirstlane(q.begin);
    q.end = __builtin_amdgcn_readfirstlane(q.end);
    return q;
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

template <int kNT>
__global__ void __launch_bounds__(kFewWaves *kWave) mx_experts_few_kernel(MxExperts g, int row_blocks)
{
    const Piece *pieces = (const Piece *)g.pieces;
    const int i = blockIdx.x / (unsigned)row_blocks;
    if (i >= piece_at(pieces, 0).expert) return;
    const Piece q = piece_at(pieces, 1 + i);
    const MxGather gather = {g.order, g.choices, g.p.n};
    few_product<kNT>(product_of(g, q.expert, q.end), (int64_t)(blockIdx.x - (unsigned)i * row_blocks) * 16, q.begin,
                     [=](int64_t at) { return gather.row_of(at); });
}

// One to four rows of X: as mx_token_kernel, a workgroup for each run of kN rows
// of a group, started by the run's first row.  Every wavefront finds the group of
// row p from the offsets itself.
template <int kN, class T>
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
    const MxGather gather = {g.order, g.choices, g.p.n};
    const int n = min(kN, end - p);
    int64_t row[kN];
#pragma unroll
    for (int t = 0; t < kN; ++t) row[t] = gather.row_of(p + min(t, n - 1));
    token_product<kN, T>(
        product_of(g, e, p + n), (int64_t)blockIdx.x * 16, p, n, d,
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
                                 MxGather{g.order, g.choices, g.p.n});
}

template <int kNT>
hipError_t launch_few(const MxExperts &g, int64_t pieces, hipStream_t s)
{
    const int64_t gx = (g.p.c + 15) / 16;
    if (!launchable(gx * pieces, kFewWaves * kWave)) return hipErrorInvalidValue;
    LaunchTimer timer(s, "mx_experts_few_kernel");
    hipLaunchKernelGGL(mx_experts_few_kernel<kNT>, dim3((unsigned)(gx * pieces)), dim3(kFewWaves * kWave), 0, s, g, (int)gx);
    return hipGetLastError();
}

template <int kTM, int kTN>
hipError_t launch_tiles(const MxExperts &g, int64_t pieces, hipStream_t s)
{
    const int64_t tiles = (g.p.c + 64 * kTM - 1) / (64 * kTM) * pieces;
    if (!launchable(tiles + kXcds - 1, 256)) return hipErrorInvalidValue;
    LaunchTimer timer(s, kTM == 2 ? (kTN == 1 ? "mx_experts_tile_kernel<2,1>" : "mx_experts_tile_kernel<2,2>")
                                  : (kTN == 2 ? "mx_experts_tile_kernel<4,2>" : "mx_experts_tile_kernel<4,4>"));
    hipLaunchKernelGGL((mx_experts_tile_kernel<kTM, kTN>), dim3((unsigned)((tiles + kXcds - 1) / kXcds * kXcds)), dim3(256),
                       0, s, g);
    return hipGetLastError();
}

template <class T>
hipError_t launch_token(const MxExperts &g, const T *X, int64_t x_ld, int d, hipStream_t s)
{
    const dim3 grid((unsigned)((g.p.c + 15) / 16), (unsigned)g.m), threads(kFewWaves * kWave);
    if (g.p.n == 1) hipLaunchKernelGGL((mx_experts_token_kernel<1, T>), grid, threads, 0, s, g, X, x_ld, d);
    else hipLaunchKernelGGL((mx_experts_token_kernel<4, T>), grid, threads, 0, s, g, X, x_ld, d);
    return hipGetLastError();
}

// How a call is done: inside one launch (rows 0), or in pieces of so many rows.
struct Way {
    int rows;
    bool few;
};

Way way_of(int64_t n, int64_t m, int64_t experts)
{
    if (mx_quantizes_inside(n) && m <= 64) return Way{0, true};
    const int64_t mean = (m + experts - 1) / experts;
    if (mean <= 16) return Way{16, true};
    if (mean <= 96) return Way{64, false};
    if (mean <= 192) return Way{128, false};
    return Way{256, false};
}

int64_t most_pieces(int64_t m, int64_t experts, int rows) { return std::min(m, m / rows + experts); }

}  // namespace

// The quantized rows of X and one of zeros, then the pieces.
size_t mx_experts_bytes(int64_t n, int64_t m, int64_t experts, int64_t d)
{
    const Way way = way_of(n, m, experts);
    if (way.rows == 0) return 0;
    const int64_t w = mx_row(d);
    return (size_t)((n + 1) * (w / 2) + ((n + 1) * (w / 32) + 15) / 16 * 16)
           + sizeof(Piece) * (size_t)(1 + most_pieces(m, experts, way.rows));
}

hipError_t launch_mx_experts(MxExperts g, const void *X, int dtype, int64_t x_ld, int64_t d, uint8_t *space, hipStream_t s)
{
    const int64_t n = g.p.n, w = mx_row(d);
    const Way way = way_of(n, g.m, g.experts);
    if (way.rows == 0) {
        if (!launchable((g.p.c + 15) / 16 * g.m, kFewWaves * kWave)) return hipErrorInvalidValue;
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
    const int64_t most = most_pieces(g.m, g.experts, way.rows);
    {
        LaunchTimer timer(s, "mx_pieces_kernel");
        hipLaunchKernelGGL(mx_pieces_kernel, dim3(1), dim3(kPieceThreads), 0, s, g.offsets, g.experts, (int)g.m, way.rows,
                           pieces, (int)most, (uint32_t *)(xc + n * (w / 2)), (uint32_t *)(xs + n * (w / 32)), g.p.nb);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const hipError_t e = launch_mx_quantize(X, dtype, n, d, x_ld, xc, xs, s);
    if (e != hipSuccess) return e;
    if (way.few) return launch_few<1>(g, most, s);
    if (way.rows == 64) return launch_tiles<2, 1>(g, most, s);
    if (way.rows == 128) return launch_tiles<2, 2>(g, most, s);
    return launch_tiles<4, 4>(g, most, s);
}

}  // namespace mpq
