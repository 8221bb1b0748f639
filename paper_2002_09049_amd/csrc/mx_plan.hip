// Pages and slots of a step's new tokens (mpq_mx_plan).
//
// Two prefix sums over the sequences: of new tokens (where a sequence's tokens
// start) and of new pages (where its pages start in the free list).  They are
// some kilobytes, so every workgroup computes them itself, kThreads sequences at
// a time, instead of waiting for another launch; then each thread looks its own
// token up in the sequences' starts in LDS.  A new page belongs to the token that
// begins it: its thread writes the table's entry.
//
// Latency bounds it: 64 sequences of one token 3.1 us, 512 sequences with 172623
// tokens 7.3 us (2.1 MB, 0.4 us of a large copy's rate).
#include "mpq.h"
#include "mx.hpp"

namespace mpq {

namespace {

// Exclusive prefix sums over the workgroup, and the sum.
template <int kThreads>
__device__ __forceinline__ int64_t prefix(int64_t v, int64_t *waves, int64_t &sum)
{
    constexpr int kWaves = kThreads / kWave;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t to = (int64_t)wave_prefix_sum((unsigned long long)v);
    if (lane == kWave - 1) waves[wave] = to;
    __syncthreads();
    int64_t before = 0;
    sum = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        if (i < wave) before += waves[i];
        sum += waves[i];
    }
    __syncthreads();
    return before + to - v;
}

template <int kThreads>
__global__ void __launch_bounds__(kThreads) mx_plan_kernel(MxPlan p)
{
    constexpr int kWaves = kThreads / kWave;
    __shared__ int64_t waves[kWaves];
    __shared__ int32_t starts[kThreads];   // of the sequences at hand
    __shared__ int32_t cached[kThreads];
    __shared__ int64_t first[kThreads];    // place in the free list of page 0, had it been new
    const int64_t token = (int64_t)blockIdx.x * kThreads + threadIdx.x, mine = (int64_t)blockIdx.x * kThreads;
    const int32_t taken = *p.taken;
    int64_t tokens = 0, pages = 0;         // of the sequences before
    bool found = false;
    for (int64_t b0 = 0; b0 < p.batch; b0 += kThreads) {
        const int64_t b = b0 + threadIdx.x;
        const int64_t old = b < p.batch ? max(p.cached[b], 0) : 0;
        int64_t fresh = b < p.batch ? max(p.fresh[b], 0) : 0, sum;
        const int64_t start = min(tokens + prefix<kThreads>(fresh, waves, sum), p.tokens);
        fresh = min(fresh, p.tokens - start);
        tokens = min(tokens + sum, p.tokens);
        const int64_t held = quotient(old + p.page - 1, p.page), need = quotient(old + fresh + p.page - 1, p.page);
        const int64_t want = max((int64_t)0, min(need, p.columns) - held);
        const int64_t at = pages + prefix<kThreads>(want, waves, sum);
        pages += sum;
        if (blockIdx.x == 0 && b < p.batch) {
            p.starts[b] = (int32_t)start;
            p.lengths[b] = (int32_t)min(old + fresh, (int64_t)0x7fffffff);
        }
        if (tokens <= mine && blockIdx.x != 0) continue;   // all of them are others' tokens
        starts[threadIdx.x] = (int32_t)start;
        cached[threadIdx.x] = (int32_t)old;
        first[threadIdx.x] = taken + at - held;
        __syncthreads();
        if (!found && token < tokens) {
            const int i = last_at_most((int)min((int64_t)kThreads, p.batch - b0), (int)token, [&](int j) { return starts[j]; });
            const int64_t position = (int64_t)cached[i] + token - starts[i], page = quotient(position, p.page);
            int32_t entry = -1;
            if (page < p.columns) {
                int32_t *in = p.table + (b0 + i) * p.table_ld + page;
                if (page * p.page < cached[i]) {
                    entry = *in;
                } else {
                    const int64_t from = first[i] + page;
                    if (from >= 0 && from < p.n_free) entry = p.free[from];
                    if (page * p.page == position) *in = entry;
                }
            }
            p.slots[token] = entry < 0 ? -1 : (int64_t)entry * p.page + (position - page * p.page);
            p.positions[token] = (int32_t)min(position, (int64_t)0x7fffffff);
            found = true;
        }
        if (tokens >= mine + kThreads && blockIdx.x != 0) return;
        __syncthreads();
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        p.starts[p.batch] = (int32_t)tokens;
        *p.taken_out = (int32_t)min(taken + pages, (int64_t)0x7fffffff);
    }
    if (!found && token < p.tokens) {
        p.slots[token] = -1;
        p.positions[token] = 0;
    }
}

}  // namespace

hipError_t launch_mx_plan(const MxPlan &p, hipStream_t s)
{
    const int threads = p.batch <= 256 ? 256 : 1024;
    const int64_t blocks = p.tokens > 0 ? (p.tokens + threads - 1) / threads : 1;
    if (!launchable(blocks, threads)) return hipErrorInvalidValue;
    LaunchTimer timer(s, "mx_plan_kernel");
    if (threads == 256) hipLaunchKernelGGL(mx_plan_kernel<256>, dim3((unsigned)blocks), dim3(256), 0, s, p);
    else hipLaunchKernelGGL(mx_plan_kernel<1024>, dim3((unsigned)blocks), dim3(1024), 0, s, p);
    return hipGetLastError();
}

}  // namespace mpq
