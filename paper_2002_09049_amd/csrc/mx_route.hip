// Routing of tokens to experts (mpq_mx_route) and the sum of their experts'
// rows (mpq_mx_combine).
//
// Routing: kLanes lanes have a token, a lane kEach consecutive experts: a whole
// wavefront for one while tokens are few (its steps are what takes time then), up
// to four tokens a wavefront where they fill the GPU (instructions are).  A logit
// is a key whose order as an unsigned number is the logits' (NaN and -infinity the
// smallest, -0 equal to 0); a 16-bit logit's key has the expert behind it.  A round
// of the choice is a maximum over the lanes; of 16-bit logits that is a choice, the
// lowest index first, of 32-bit ones the first lane that holds it, and there the first
// key, is.  The softmax statistics are fp32.  16384 tokens, 256 experts, 8 choices:
// 9.0 us (bf16) and 12.2 us (fp32), by a wavefront a token 19.6 us; 200 tokens, 300
// experts, 10 choices, fp32: 7.7 us by a wavefront a token, by half a one 18.5.  Sorting
// a lane's four largest first, so that a round touches only those, took 10.0 and 13.1 us:
// the steps of a round over the lanes are most of it.
//
// The choices are then sorted by expert, tokens in order: of a workgroup's 64
// tokens an expert has a mask of 64 bits in LDS (set by "or", whose order does not
// matter), and a choice's rank among the workgroup's choices of its expert is
// the number of bits below its token's.  What the workgroups before have chosen
// is added up from their counts, a byte each, by a second kernel; where that
// would have every workgroup read too many, a kernel between the two does it
// once.  Up to 64 tokens one workgroup, and one launch, do it all.
#include <algorithm>
#include <type_traits>

#include "mpq.h"
#include "mx.hpp"

namespace mpq {

namespace {

constexpr int kThreads = 1024;
constexpr int kMostExperts = 1024;

// Tokens of a workgroup: a wavefront's each, or as many as a mask has bits.
constexpr int64_t kFew = 4096;
__host__ __device__ __forceinline__ int tokens_of(int64_t n) { return n > 64 && n <= kFew ? 16 : 64; }

// Bytes of a workgroup's counts.
__host__ __device__ __forceinline__ int pitch_of(int experts) { return (experts + 3) / 4 * 4; }

// Maximum, minimum or sum over the kLanes lanes of a token.
template <int kLanes, class V, class Op>
__device__ __forceinline__ V lanes_reduce(V v, Op op)
{
    v = op(v, xstep<0>(v));
    v = op(v, xstep<1>(v));
    v = op(v, xstep<2>(v));
    v = op(v, xstep<3>(v));
    if constexpr (kLanes >= 32) {
        V a, b;
        swap_step<false>(v, a, b);
        v = op(a, b);
    }
    if constexpr (kLanes >= 64) {
        V a, b;
        swap_step<true>(v, a, b);
        v = op(a, b);
    }
    return v;
}

// The order of a logit; 0 is below all.
__device__ __forceinline__ uint32_t order_of(float v)
{
    if (!(v > -INFINITY)) return 0x007fffffu;   // -infinity's
    const uint32_t u = __float_as_uint(v + 0.0f);
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t order)
{
    return __uint_as_float(order >> 31 ? order & 0x7fffffffu : ~order);
}
// The same of 16 bits.
template <class T>
__device__ __forceinline__ uint32_t order16_of(T v)
{
    if (!((float)v > -INFINITY)) v = (T)-INFINITY;
    if ((float)v == 0.0f) v = (T)0.0f;
    uint16_t u;
    __builtin_memcpy(&u, &v, 2);
    return u >> 15 ? (uint16_t)~u : u | 0x8000u;
}
template <class T>
__device__ __forceinline__ float value16_of(uint32_t order)
{
    const uint16_t u = (uint16_t)(order >> 15 ? order & 0x7fffu : ~order);
    T v;
    __builtin_memcpy(&v, &u, 2);
    return (float)v;
}

// A lane's keys.
template <class T, int kLanes, int kEach>
struct Keys {
    static constexpr bool kAlone = std::is_same_v<T, float>;   // a key is the order alone
    uint32_t key[kEach], most;

    __device__ __forceinline__ void largest()
    {
        most = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) most = max(most, key[i]);
    }
    __device__ __forceinline__ void load(const T *row, int first, int experts)
    {
        T v[kEach];
        if constexpr (kEach % 8 == 0) {
#pragma unroll
            for (int i = 0; i < kEach; i += 8) {
                const Eight<T> e = load_eight(row + first + i, experts - first - i);
                __builtin_memcpy(v + i, e.w, sizeof e.w);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kEach; ++i) v[i] = first + i < experts ? row[first + i] : (T)0.0f;
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if constexpr (kAlone) key[i] = order_of(v[i]);
            else key[i] = order16_of(v[i]) << 16 | (uint32_t)(0xffff - (first + i));
            if (first + i >= experts) key[i] = 0;
        }
        largest();
    }
    __device__ __forceinline__ float value(uint32_t k) const
    {
        if constexpr (kAlone) return value_of(k);
        else return value16_of<T>(k >> 16);
    }
    // The largest of all lanes, taken out; its expert to *expert.
    __device__ __forceinline__ uint32_t take(int first, uint16_t *expert)
    {
        const uint32_t best = lanes_reduce<kLanes>(most, MaxOp());
        if constexpr (kAlone) {
            const unsigned long long have = __ballot(most == best);
            unsigned first_lane;
            if constexpr (kLanes == 64) first_lane = (unsigned)__builtin_ctzll(have);
            else first_lane = (unsigned)__builtin_ctz((uint32_t)(have >> (threadIdx.x % kWave / kLanes * kLanes)));
            const bool winner = threadIdx.x % kLanes == first_lane;
            bool open = winner;
            int at = 0;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const bool taken = open && key[i] == best;
                at = taken ? i : at;
                key[i] = taken ? 0u : key[i];
                open = open && !taken;
            }
            if (winner) *expert = (uint16_t)(first + at);
        } else {
            if (first == 0) *expert = (uint16_t)(0xffff - (best & 0xffff));
#pragma unroll
            for (int i = 0; i < kEach; ++i) key[i] = key[i] == best ? 0u : key[i];
        }
        largest();
        return best;
    }
};

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

// kAlone: this workgroup has all tokens.
template <int kLanes, int kEach, bool kAlone, class T>
__global__ void __launch_bounds__(kThreads) mx_choose_kernel(MxRoute r, int of_block)
{
    __shared__ unsigned long long masks[kMostExperts];
    __shared__ uint32_t counts[kMostExperts + 1];
    __shared__ uint16_t taken[kThreads];   // a lane each: its token's choice of that number
    const int lane = threadIdx.x % kLanes, first = lane * kEach;
    uint16_t *choices = taken + (threadIdx.x - lane);
    for (int e = threadIdx.x; e < r.experts; e += kThreads) masks[e] = 0;
    __syncthreads();
    const int64_t token0 = (int64_t)blockIdx.x * of_block;
    const int tokens = (int)min((int64_t)of_block, r.n - token0);
    for (int t = threadIdx.x / kLanes; t < tokens; t += kThreads / kLanes) {
        Keys<T, kLanes, kEach> keys;
        keys.load((const T *)r.logits + (token0 + t) * r.ld, first, r.experts);
        float all = 0.0f, top = 0.0f, mine = 0.0f;
        if (!r.renorm) {
            top = keys.value(lanes_reduce<kLanes>(keys.most, MaxOp()));
#pragma unroll
            for (int i = 0; i < kEach; ++i) all += keys.key[i] ? part_of(keys.value(keys.key[i]), top) : 0.0f;
            all = lanes_reduce<kLanes>(all, SumOp());
        }
        for (int j = 0; j < r.k; ++j) {
            const float v = keys.value(keys.take(first, choices + j));
            if (j == 0) top = v;
            if (lane == j) mine = v;
        }
        mine = lane < r.k ? part_of(mine, top) : 0.0f;
        if (r.renorm) all = lanes_reduce<kLanes>(mine, SumOp());
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (lane < r.k) {
            const int chosen = choices[lane];
            const int64_t at = (token0 + t) * r.k + lane;
            r.chosen[at] = chosen;
            r.weights[at] = all > 0.0f ? mine / all : 0.0f;
            atomicOr(&masks[chosen], 1ull << t);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
    if constexpr (kAlone) {
        for (int e = threadIdx.x; e < r.experts; e += kThreads) counts[e] = (uint32_t)__popcll(masks[e]);
        prefix_counts(counts, r.experts);
        for (int e = threadIdx.x; e <= r.experts; e += kThreads) r.offsets[e] = (int32_t)counts[e];
    } else {
        const int pitch = pitch_of(r.experts);
        for (int e = threadIdx.x; e < pitch; e += kThreads)
            r.counts[(int64_t)blockIdx.x * pitch + e] = e < r.experts ? (uint8_t)__popcll(masks[e]) : 0;
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

// Every workgroup's counts to sums [blocks][experts] of the workgroups before it,
// and the sums of all behind them (row `blocks`).  A workgroup has 16 experts and
// 64 runs of rows.
constexpr int kColumns = 16, kRuns = kThreads / kColumns;
__global__ void __launch_bounds__(kThreads) mx_sum_kernel(const uint8_t *counts, int32_t *to, int blocks, int experts)
{
    __shared__ int32_t sums[kRuns][kColumns];
    const int column = threadIdx.x % kColumns, run = threadIdx.x / kColumns, e = blockIdx.x * kColumns + column;
    const int each = (blocks + kRuns - 1) / kRuns, from = min(run * each, blocks), end = min(from + each, blocks);
    const int pitch = pitch_of(experts);
    int32_t sum = 0;
    if (e < experts)
#pragma unroll 8
        for (int b = from; b < end; ++b) sum += counts[(int64_t)b * pitch + e];
    sums[run][column] = sum;
    __syncthreads();
    if (e >= experts) return;
    int32_t before = 0;
    for (int i = 0; i < run; ++i) before += sums[i][column];
#pragma unroll 8
    for (int b = from; b < end; ++b) {
        to[(int64_t)b * experts + e] = before;
        before += counts[(int64_t)b * pitch + e];
    }
    if (run == kRuns - 1) to[(int64_t)blocks * experts + e] = before;
}

// Each choice to its place.  kSummed: by mx_sum_kernel's sums; else this workgroup
// adds up the counts itself, four experts a word: pairs of 16-bit sums, which
// hold up to 1023 rows of 64.  A word's rows are shared by up to kMostParts threads,
// whose sums a thread an expert then adds one by one: as many as the workgroup
// has threads for, and sums of no rows among them, took 21.6 us for 2 or 4 experts and 12.5
// for 8, at 100 tokens or 16384, where 32 take 3.5 to 5.0 (16: as long, but 60000 tokens
// of 8 experts 10.3 and 9.0; 64: 0.2 to 0.6 more).
constexpr int kMostAdded = 1023, kMostParts = 32;
template <bool kSummed>
__global__ void __launch_bounds__(kThreads) mx_place_kernel(MxRoute r, int blocks, int of_block)
{
    __shared__ uint32_t counts[kMostExperts + 1], before[kMostExperts];
    if constexpr (kSummed) {
        for (int e = threadIdx.x; e < r.experts; e += kThreads) {
            counts[e] = (uint32_t)r.sums[(int64_t)blocks * r.experts + e];
            before[e] = (uint32_t)r.sums[(int64_t)blockIdx.x * r.experts + e];
        }
    } else {
        // two words of pairs for the rows before, two for all
        __shared__ uint32_t part[4][kThreads];
        const int words = pitch_of(r.experts) / 4, runs = min(min(kThreads / words, kMostParts), blocks);
        const int word = threadIdx.x % words, run = threadIdx.x / words, here = blockIdx.x;
        uint32_t even = 0, odd = 0, even_before = 0, odd_before = 0;
        if (run < runs) {
            const uint32_t *from = (const uint32_t *)r.counts + word;
            int b = run;
#pragma unroll 8
            for (; b < here; b += runs) {
                const uint32_t v = from[(int64_t)b * words];
                even += v & 0x00ff00ffu;
                odd += v >> 8 & 0x00ff00ffu;
            }
            even_before = even;
            odd_before = odd;
#pragma unroll 8
            for (; b < blocks; b += runs) {
                const uint32_t v = from[(int64_t)b * words];
                even += v & 0x00ff00ffu;
                odd += v >> 8 & 0x00ff00ffu;
            }
        }
        part[0][threadIdx.x] = even;
        part[1][threadIdx.x] = odd;
        part[2][threadIdx.x] = even_before;
        part[3][threadIdx.x] = odd_before;
        __syncthreads();
        for (int e = threadIdx.x; e < r.experts; e += kThreads) {
            uint32_t all = 0, some = 0;
            for (int i = 0; i < runs; ++i) {
                const int at = i * words + e / 4, shift = e % 4 / 2 * 16;
                all += part[e % 2][at] >> shift & 0xffffu;
                some += part[2 + e % 2][at] >> shift & 0xffffu;
            }
            counts[e] = all;
            before[e] = some;
        }
    }
    prefix_counts(counts, r.experts);
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= r.experts; e += kThreads) r.offsets[e] = (int32_t)counts[e];
    const int64_t token0 = (int64_t)blockIdx.x * of_block;
    const int tokens = (int)min((int64_t)of_block, r.n - token0);
    for (int i = threadIdx.x; i < tokens * r.k; i += kThreads) {
        const int64_t at = token0 * r.k + i;
        const int e = r.chosen[at];
        const int32_t to = (int32_t)(counts[e] + before[e]) + r.place[at];
        r.place[at] = to;
        r.order[to] = (int32_t)at;
    }
}

// A wavefront a token.
template <bool kAlone, class T>
auto choose_wide(int experts)
{
    return experts <= 64    ? mx_choose_kernel<64, 1, kAlone, T>
           : experts <= 128 ? mx_choose_kernel<64, 2, kAlone, T>
           : experts <= 256 ? mx_choose_kernel<64, 4, kAlone, T>
           : experts <= 512 ? mx_choose_kernel<64, 8, kAlone, T>
                            : mx_choose_kernel<64, 16, kAlone, T>;
}

template <class T>
hipError_t choose_as(const MxRoute &r, int64_t blocks, hipStream_t s)
{
    const int of_block = tokens_of(r.n);
    auto kern = blocks <= 1 ? choose_wide<true, T>(r.experts) : choose_wide<false, T>(r.experts);
    if (of_block == 64 && blocks > 1 && r.k <= 16) {   // a choice is kept by the lane of its number
        if (r.experts <= 16) kern = mx_choose_kernel<16, 1, false, T>;
        else if (r.experts <= 64) kern = mx_choose_kernel<16, 4, false, T>;
        else if (r.experts <= 128) kern = mx_choose_kernel<16, 8, false, T>;
        else if (r.experts <= 256) kern = mx_choose_kernel<16, 16, false, T>;
        else if (r.experts <= 512) kern = mx_choose_kernel<32, 16, false, T>;
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)std::max((int64_t)1, blocks)), dim3(kThreads), 0, s, r, of_block);
    return hipGetLastError();
}

hipError_t choose(const MxRoute &r, int64_t blocks, hipStream_t s)
{
    LaunchTimer timer(s, "mx_choose_kernel");
    if (r.dtype == MPQ_F32) return choose_as<float>(r, blocks, s);
    if (r.dtype == MPQ_F16) return choose_as<_Float16>(r, blocks, s);
    return choose_as<__bf16>(r, blocks, s);
}

int64_t blocks_of(int64_t n) { return (n + tokens_of(n) - 1) / tokens_of(n); }

// Whether the workgroups add up the counts themselves: while all of them together
// read few (16384 tokens, 256 experts: 6.4 us; with mx_sum_kernel before, which has
// to be waited for, 4.4 + 4.2; 65536 tokens, 128 experts by that 6.3 + 7.0;
// 60000 of 32 experts inside 9.7, of 64 by that 6.9 + 4.5).
bool adds_inside(int64_t blocks, int64_t experts)
{
    return blocks <= kMostAdded && blocks * blocks * pitch_of((int)experts) <= (int64_t)32 << 20;
}

size_t count_bytes(int64_t blocks, int64_t experts) { return (size_t)((blocks * pitch_of((int)experts) + 15) / 16 * 16); }

// A thread has eight columns of a token.  Memory bounds it: k rows are read for
// one that is written (8192 tokens, 8 rows of 2048, bf16: 68 us, 4.9 TB/s).
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
    const int64_t blocks = blocks_of(n);
    if (blocks <= 1) return 0;
    const size_t bytes = count_bytes(blocks, experts)
                         + (adds_inside(blocks, experts) ? 0 : (size_t)((blocks + 1) * experts) * sizeof(int32_t));
    // (a little past kFew workgroups are fewer: not below what fewer tokens take)
    return n > kFew ? std::max(bytes, mx_route_bytes(kFew, experts)) : bytes;
}

hipError_t launch_mx_route(MxRoute r, void *space, hipStream_t s)
{
    const int64_t blocks = blocks_of(r.n);
    const int of_block = tokens_of(r.n);
    if (blocks <= 1) return choose(r, blocks, s);
    r.counts = (uint8_t *)space;
    r.sums = (int32_t *)((uint8_t *)space + count_bytes(blocks, r.experts));
    hipError_t e = choose(r, blocks, s);
    if (e != hipSuccess) return e;
    if (adds_inside(blocks, r.experts)) {
        LaunchTimer timer(s, "mx_place_kernel");
        hipLaunchKernelGGL(mx_place_kernel<false>, dim3((unsigned)blocks), dim3(kThreads), 0, s, r, (int)blocks, of_block);
        return hipGetLastError();
    }
    {
        LaunchTimer timer(s, "mx_sum_kernel");
        hipLaunchKernelGGL(mx_sum_kernel, dim3((unsigned)(r.experts + kColumns - 1) / kColumns), dim3(kThreads), 0, s,
                           r.counts, r.sums, (int)blocks, r.experts);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    LaunchTimer timer(s, "mx_place_kernel");
    hipLaunchKernelGGL(mx_place_kernel<true>, dim3((unsigned)blocks), dim3(kThreads), 0, s, r, (int)blocks, of_block);
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
