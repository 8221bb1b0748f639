// Keys and values into the pages of a block-scaled cache and back
// (mpq_mx_cache_write, mpq_mx_cache_read).
//
// A row is the head_dim values of one token and head; it is held as nb =
// ceil(head_dim / 32) blocks.  A thread holds eight consecutive elements, so a
// row takes 4 nb threads and a quad holds a block, as in mx_quantize.hip; the
// grid's second dimension chooses keys or values.  In the cache a head's rows
// of one page follow each other, and their scales are stored block by block,
// consecutive tokens' scales of one block beside each other: attention reads
// four tokens' scales as one word.
#include "mpq.h"
#include "mx.hpp"

namespace mpq {

namespace {

constexpr int kThreads = 256;

struct Place {
    int64_t token;
    int head, j;      // j: first of the eight elements in the row
};

__device__ __forceinline__ Place place(int heads, int nb)
{
    const uint32_t per = 4u * (uint32_t)nb;   // threads a row
    const int64_t first = (int64_t)blockIdx.x * kThreads;
    const int64_t row0 = first / per;
    const uint32_t off = (uint32_t)(first - row0 * per) + threadIdx.x;
    const int64_t token0 = row0 / heads;
    const uint32_t h = (uint32_t)(row0 - token0 * heads) + off / per;
    Place p;
    p.token = token0 + h / (uint32_t)heads;
    p.head = (int)(h % (uint32_t)heads);
    p.j = (int)(off % per) * 8;
    return p;
}

// Where a slot is: page and the token's place in it.
__device__ __forceinline__ void find(const MxCacheView &c, int64_t slot, int64_t &page, int &at)
{
    if (slot < 0x80000000LL) {
        page = (uint32_t)slot / (uint32_t)c.page;
        at = (int)((uint32_t)slot % (uint32_t)c.page);
    } else {
        page = slot / c.page;
        at = (int)(slot - page * c.page);
    }
}

template <int kFmt, class T>
__global__ void __launch_bounds__(kThreads) mx_cache_write_kernel(MxCacheView c, const T *K, const T *V, int64_t k_tok,
                                                                  int64_t k_head, int64_t v_tok, int64_t v_head,
                                                                  int64_t tokens, const int64_t *slots)
{
    const Place p = place(c.heads, c.nb);
    if (p.token >= tokens) return;
    const int64_t slot = slots[p.token];
    if (slot < 0 || slot >= c.n_pages * c.page) return;
    int64_t page;
    int at;
    find(c, slot, page, at);
    const bool val = blockIdx.y != 0;
    const T *x0 = val ? V + p.token * v_tok + p.head * v_head : K + p.token * k_tok + p.head * k_head;
    float x[8];
    load8(x0 + p.j, c.dim - p.j, x);
    const uint32_t s = mx_scale_byte<kFmt>(quad_max(largest_bits(x)));
    constexpr int kWords = kFmt == kFp4 ? 1 : 2;
    uint32_t w[kWords];
    mx_codes<kFmt>(x, s, w);
    const int64_t ph = page * c.heads + p.head;
    uint8_t *codes = (val ? c.v : c.k) + (ph * c.page + at) * (c.nb * 16 * kWords) + p.j / 2 * kWords;
    __builtin_memcpy(__builtin_assume_aligned(codes, 4 * kWords), w, sizeof w);
    if (p.j % kMxBlock == 0) (val ? c.vs : c.ks)[(ph * c.nb + p.j / kMxBlock) * c.page + at] = (uint8_t)s;
}

template <int kFmt, class T>
__global__ void __launch_bounds__(kThreads) mx_cache_read_kernel(MxCacheView c, T *K, T *V, int64_t k_tok,
                                                                 int64_t k_head, int64_t v_tok, int64_t v_head,
                                                                 int64_t tokens, const int64_t *slots)
{
    const Place p = place(c.heads, c.nb);
    if (p.token >= tokens || p.j >= c.dim) return;
    const bool val = blockIdx.y != 0;
    T *y = (val ? V + p.token * v_tok + p.head * v_head : K + p.token * k_tok + p.head * k_head) + p.j;
    const int64_t slot = slots[p.token];
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (slot >= 0 && slot < c.n_pages * c.page) {
        int64_t page;
        int at;
        find(c, slot, page, at);
        constexpr int kWords = kFmt == kFp4 ? 1 : 2;
        const int64_t ph = page * c.heads + p.head;
        const uint8_t *codes = (val ? c.v : c.k) + (ph * c.page + at) * (c.nb * 16 * kWords) + p.j / 2 * kWords;
        uint32_t w[kWords];
        __builtin_memcpy(w, __builtin_assume_aligned(codes, 4 * kWords), sizeof w);
        mx_values<kFmt>(w, (val ? c.vs : c.ks)[(ph * c.nb + p.j / kMxBlock) * c.page + at], x);
    }
    store8(y, c.dim - p.j, x);
}

int64_t row_blocks(const MxCacheView &c, int64_t tokens)
{
    // tokens * heads * nb is below 2^62 (host checks on each)
    return (tokens * c.heads * c.nb * 4 + kThreads - 1) / kThreads;
}

}  // namespace

template <class T>
static hipError_t write_as(const MxCacheView &c, const MxRows &r, int64_t tokens, const int64_t *slots, unsigned blocks,
                           hipStream_t s)
{
    auto kern = c.fmt == kFp4 ? mx_cache_write_kernel<kFp4, T> : mx_cache_write_kernel<kFp8, T>;
    hipLaunchKernelGGL(kern, dim3(blocks, 2), dim3(kThreads), 0, s, c, (const T *)r.K, (const T *)r.V, r.k_tok,
                       r.k_head, r.v_tok, r.v_head, tokens, slots);
    return hipGetLastError();
}

template <class T>
static hipError_t read_as(const MxCacheView &c, const MxRows &r, int64_t tokens, const int64_t *slots, unsigned blocks,
                          hipStream_t s)
{
    auto kern = c.fmt == kFp4 ? mx_cache_read_kernel<kFp4, T> : mx_cache_read_kernel<kFp8, T>;
    hipLaunchKernelGGL(kern, dim3(blocks, 2), dim3(kThreads), 0, s, c, (T *)r.K, (T *)r.V, r.k_tok, r.k_head, r.v_tok,
                       r.v_head, tokens, slots);
    return hipGetLastError();
}

hipError_t launch_mx_cache_write(const MxCacheView &c, const MxRows &r, int64_t tokens, const int64_t *slots,
                                 hipStream_t s)
{
    const int64_t blocks = row_blocks(c, tokens);
    if (blocks <= 0) return hipSuccess;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
    LaunchTimer timer(s, "mx_cache_write_kernel");
    if (r.dtype == MPQ_F32) return write_as<float>(c, r, tokens, slots, (unsigned)blocks, s);
    if (r.dtype == MPQ_F16) return write_as<_Float16>(c, r, tokens, slots, (unsigned)blocks, s);
    return write_as<__bf16>(c, r, tokens, slots, (unsigned)blocks, s);
}

hipError_t launch_mx_cache_read(const MxCacheView &c, const MxRows &r, int64_t tokens, const int64_t *slots,
                                hipStream_t s)
{
    const int64_t blocks = row_blocks(c, tokens);
    if (blocks <= 0) return hipSuccess;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
    LaunchTimer timer(s, "mx_cache_read_kernel");
    if (r.dtype == MPQ_F32) return read_as<float>(c, r, tokens, slots, (unsigned)blocks, s);
    if (r.dtype == MPQ_F16) return read_as<_Float16>(c, r, tokens, slots, (unsigned)blocks, s);
    return read_as<__bf16>(c, r, tokens, slots, (unsigned)blocks, s);
}

}  // namespace mpq
