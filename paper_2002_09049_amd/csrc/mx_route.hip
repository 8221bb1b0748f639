// Routing of tokens to experts (mpq_mx_route) and the sum of their experts'
// rows (mpq_mx_combine).
//
// Routing: a wavefront has a token, a lane a run of consecutive experts.  A
// logit is a 32-bit key whose order as an unsigned number is the logits' (NaN
// and -infinity the smallest, -0 equal to 0), so a round of the choice is one
// maximum over the lanes and a ballot, whose first lane, and there the first
// key, is the choice of the lowest index.  The softmax statistics are fp32.
//
// The choices are then sorted by expert, tokens in order: of a workgroup's 64
// tokens an expert has a mask of 64 bits in LDS (set by "or", whose order does not
// matter), and a choice's rank among the workgroup's choices of its expert is
// the number of bits below its token's.  What the workgroups before have chosen
// is added up by a second kernel (experts in parallel), and a third puts each
// choice in its place.  Up to 64 tokens one workgroup, and one launch, do it all.
#include <algorithm>

#include "mpq.h"
#include "mx.hpp"

namespace mpq {

namespace {

constexpr int kTokens = 64;       // of a workgroup
constexpr int kThreads = 1024;
constexpr int kMostExperts = 1024;

__device__ __forceinline__ uint32_t key_of(float v)
{
    if (!(v > -INFINITY)) return 0x007fffffu;   // -infinity's
    const uint32_t u = __float_as_uint(v + 0.0f);
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key)
{
    return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key);
}
// exp(v - top), an infinite top's equals included
__device__ __forceinline__ float part_of(float v, float top)
{
    return top == -INFINITY ? 0.0f : v == top ? 1.0f : expf(v - top);
}

// Exclusive prefix sums of counts[0 .. experts) in LDS by the first wavefront,
// counts[experts] the sum.  The workgroup meets before and after.
__device__ __forceinline__ void prefix_counts(uint32_t *counts, int experts)
{
    __syncthreads();
    if (threadIdx.x < kWave) {
        const int lane = threadIdx.x, each = (experts + kWave - 1) / kWave;
        uint32_t sum = 0;
        for (int i = 0; i < each; ++i) sum += lane * each + i < experts ? counts[lane * each + i] : 0;
        uint32_t before = wave_prefix_sum(sum) - sum;
        for (int i = 0; i < each; ++i) {
            if (lane * each + i >= experts) break;
            const uint32_t c = counts[lane * each + i];
            counts[lane * each + i] = before;
            before += c;
        }
        if (lane == kWave - 1) counts[experts] = before;
    }
    __syncthreads();
}

// kEach: experts of a lane.  kAlone: this workgroup has all tokens.
template <int kEach, bool kAlone, class T>
__global__ void __launch_bounds__(kThreads) mx_choose_kernel(MxRoute r)
{
    __shared__ unsigned long long masks[kMostExperts];
    __shared__ uint32_t counts[kMostExperts + 1];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    for (int e = threadIdx.x; e < r.experts; e += kThreads) masks[e] = 0;
    __syncthreads();
    const int64_t token0 = (int64_t)blockIdx.x * kTokens;
    const int tokens = (int)min((int64_t)kTokens, r.n - token0);
    for (int t = wave; t < tokens; t += kThreads / kWave) {
        const T *row = (const T *)r.logits + (token0 + t) * r.ld;
        uint32_t key[kEach], most = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int e = lane * kEach + i;
            key[i] = e < r.experts ? key_of((float)row[e]) : 0u;
            most = max(most, key[i]);
        }
        float all = 0.0f, top = 0.0f, mine = 0.0f;
        int chosen = 0;
        for (int j = 0; j < r.k; ++j) {
            const uint32_t best = wave_reduce(most, MaxOp());
            const int winner = __builtin_ctzll(__ballot(most == best));
            int e = 0;
#pragma unroll
            for (int i = kEach - 1; i >= 0; --i) e = key[i] == best ? i : e;
            e = readlane(e, winner);
            if (j == 0) {
                top = value_of(best);
                if (!r.renorm) {
#pragma unroll
                    for (int i = 0; i < kEach; ++i) all += key[i] ? part_of(value_of(key[i]), top) : 0.0f;
                    all = wave_reduce(all, SumOp());
                }
            }
            if (lane == j) {
                chosen = winner * kEach + e;
                mine = part_of(value_of(best), top);
            }
            most = 0;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                if (lane == winner && i == e) key[i] = 0;
                most = max(most, key[i]);
            }
        }
        if (r.renorm) all = wave_reduce(mine, SumOp());
        if (lane < r.k) {
            const int64_t at = (token0 + t) * r.k + lane;
            r.chosen[at] = chosen;
            r.weights[at] = all > 0.0f ? mine / all : 0.0f;
            atomicOr(&masks[chosen], 1ull << t);
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < r.experts; e += kThreads) {
        const uint32_t c = (uint32_t)__popcll(masks[e]);
        if constexpr (kAlone) counts[e] = c;
        else r.counts[(int64_t)blockIdx.x * r.experts + e] = (int32_t)c;
    }
    if constexpr (kAlone) {
        prefix_counts(counts, r.experts);
        for (int e = threadIdx.x; e <= r.experts; e += kThreads) r.offsets[e] = (int32_t)counts[e];
    }
    for (int i = threadIdx.x; i < tokens * r.k; i += kThreads) {
        const int64_t at = token0 * r.k + i;
        const int e = r.chosen[at], t = i / r.k;   // written by this workgroup, before the barrier
        const int rank = __popcll(masks[e] & ((1ull << t) - 1));
        if constexpr (kAlone) {
            r.place[at] = (int32_t)counts[e] + rank;
            r.order[counts[e] + rank] = (int32_t)at;
        } else {
            r.place[at] = rank;
        }
    }
}

// counts [blocks][experts] to their exclusive sums over the blocks, the sums
// behind them (row `blocks`).  A workgroup has 16 experts and 64 runs of blocks.
constexpr int kColumns = 16, kRuns = kThreads / kColumns;
__global__ void __launch_bounds__(kThreads) mx_sum_kernel(int32_t *counts, int blocks, int experts)
{
    __shared__ int32_t sums[kRuns][kColumns];
    const int column = threadIdx.x % kColumns, run = threadIdx.x / kColumns, e = blockIdx.x * kColumns + column;
    const int each = (blocks + kRuns - 1) / kRuns, from = min(run * each, blocks), to = min(from + each, blocks);
    int32_t sum = 0;
    if (e < experts)
        for (int b = from; b < to; ++b) sum += counts[(int64_t)b * experts + e];
    sums[run][column] = sum;
    __syncthreads();
    if (e >= experts) return;
    int32_t before = 0;
    for (int i = 0; i < run; ++i) before += sums[i][column];
    for (int b = from; b < to; ++b) {
        int32_t *c = counts + (int64_t)b * experts + e;
        const int32_t v = *c;
        *c = before;
        before += v;
    }
    if (run == kRuns - 1) counts[(int64_t)blocks * experts + e] = before;
}

__global__ void __launch_bounds__(256) mx_place_kernel(MxRoute r, int blocks)
{
    __shared__ uint32_t counts[kMostExperts + 1];
    for (int e = threadIdx.x; e < r.experts; e += 256) counts[e] = (uint32_t)r.counts[(int64_t)blocks * r.experts + e];
    prefix_counts(counts, r.experts);
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= r.experts; e += 256) r.offsets[e] = (int32_t)counts[e];
    const int64_t token0 = (int64_t)blockIdx.x * kTokens;
    const int tokens = (int)min((int64_t)kTokens, r.n - token0);
    const int32_t *before = r.counts + (int64_t)blockIdx.x * r.experts;
    for (int i = threadIdx.x; i < tokens * r.k; i += 256) {
        const int64_t at = token0 * r.k + i;
        const int e = r.chosen[at];
        const int32_t to = (int32_t)counts[e] + before[e] + r.place[at];
        r.place[at] = to;
        r.order[to] = (int32_t)at;
    }
}

template <bool kAlone, class T>
hipError_t choose_as(const MxRoute &r, unsigned blocks, hipStream_t s)
{
    auto kern = r.experts <= 64    ? mx_choose_kernel<1, kAlone, T>
                : r.experts <= 128 ? mx_choose_kernel<2, kAlone, T>
                : r.experts <= 256 ? mx_choose_kernel<4, kAlone, T>
                : r.experts <= 512 ? mx_choose_kernel<8, kAlone, T>
                                   : mx_choose_kernel<16, kAlone, T>;
    hipLaunchKernelGGL(kern, dim3(blocks), dim3(kThreads), 0, s, r);
    return hipGetLastError();
}

template <bool kAlone>
hipError_t choose(const MxRoute &r, unsigned blocks, hipStream_t s)
{
    LaunchTimer timer(s, "mx_choose_kernel");
    if (r.dtype == MPQ_F32) return choose_as<kAlone, float>(r, blocks, s);
    if (r.dtype == MPQ_F16) return choose_as<kAlone, _Float16>(r, blocks, s);
    return choose_as<kAlone, __bf16>(r, blocks, s);
}

// A thread has eight columns of a token.  Memory bounds it: k rows are read for
// one that is written.
template <class T, class Z>
__global__ void __launch_bounds__(256) mx_combine_kernel(MxCombine q, int chunks)
{
    const int64_t item = block_of(blockIdx.y) * 256 + threadIdx.x, token = quotient(item, chunks);
    if (token >= q.n) return;
    const int64_t col = (item - token * chunks) * 8;
    const int live = (int)min((int64_t)8, q.c - col);
    float z[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (q.R) load8((const T *)q.R + token * q.ldr + col, live, z);
    const int32_t *place = q.place + token * q.k;
    const float *weight = q.weights + token * q.k;
    for (int j = 0; j < q.k; ++j) {
        const int64_t row = place[j];
        if (row < 0 || row >= q.m) continue;
        const float w = weight[j];
        float y[8];
        load8((const T *)q.Y + row * q.ldy + col, live, y);
#pragma unroll
        for (int v = 0; v < 8; ++v) z[v] += w * y[v];
    }
    store8<false>((Z *)q.Z + token * q.ldz + col, live, z);
}

template <class T>
hipError_t combine_as(const MxCombine &q, int chunks, dim3 grid, hipStream_t s)
{
    auto kern = q.z_dtype == MPQ_F32   ? mx_combine_kernel<T, float>
                : q.z_dtype == MPQ_F16 ? mx_combine_kernel<T, _Float16>
                                       : mx_combine_kernel<T, __bf16>;
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, q, chunks);
    return hipGetLastError();
}

}  // namespace

size_t mx_route_bytes(int64_t n, int64_t experts)
{
    const int64_t blocks = (n + kTokens - 1) / kTokens;
    return blocks <= 1 ? 0 : (size_t)((blocks + 1) * experts) * sizeof(int32_t);
}

hipError_t launch_mx_route(const MxRoute &r, hipStream_t s)
{
    const unsigned blocks = (unsigned)((r.n + kTokens - 1) / kTokens);
    if (blocks <= 1) return choose<true>(r, 1, s);
    hipError_t e = choose<false>(r, blocks, s);
    if (e != hipSuccess) return e;
    {
        LaunchTimer timer(s, "mx_sum_kernel");
        hipLaunchKernelGGL(mx_sum_kernel, dim3((unsigned)(r.experts + kColumns - 1) / kColumns), dim3(kThreads), 0, s,
                           r.counts, (int)blocks, r.experts);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    LaunchTimer timer(s, "mx_place_kernel");
    hipLaunchKernelGGL(mx_place_kernel, dim3(blocks), dim3(256), 0, s, r, (int)blocks);
    return hipGetLastError();
}

hipError_t launch_mx_combine(const MxCombine &q, hipStream_t s)
{
    const int64_t chunks = (q.c + 7) / 8, blocks = (q.n * chunks + 255) / 256;
    if (blocks <= 0) return hipSuccess;
    if (grid_rows(blocks) > 65535) return hipErrorInvalidValue;
    const dim3 grid(grid_x(blocks), (unsigned)grid_rows(blocks));
    LaunchTimer timer(s, "mx_combine_kernel");
    if (q.dtype == MPQ_F32) return combine_as<float>(q, (int)chunks, grid, s);
    if (q.dtype == MPQ_F16) return combine_as<_Float16>(q, (int)chunks, grid, s);
    return combine_as<__bf16>(q, (int)chunks, grid, s);
}

}  // namespace mpq
