// Keys and values into the pages of a block-scaled cache and back
// (mpq_mx_cache_write, mpq_mx_cache_read).
//
// A row is the head_dim values of one token and head; it is held as nb =
// ceil(head_dim / 32) blocks.  A thread holds eight consecutive elements of a
// key's row and the same of the value's, so a row takes 4 nb threads and a
// quad holds a block, as in mx_quantize.hip; a workgroup takes as many whole
// rows as fit its 256 threads.  Memory bounds both, once the places are found
// without divisions of large numbers (with them: 52 and 45 us for 32768 tokens
// of 8 heads of 128 in fp4; without, 39 and 34 us, 4.4 and 5.0 TB/s of the 170 MB
// that either moves).  Writing is the slower: tokens at slots in any order fill
// parts of lines (63 MB written for the 36 MB held).
//
// In the cache a head's rows of one page follow each other, and their scales
// are stored block by block, consecutive tokens' scales of one block beside
// each other: attention reads four tokens' scales as one word.
#include "mpq.h"
#include "mx_cache.hpp"

namespace mpq {

namespace {

constexpr int kThreads = 256;

// Rows of a workgroup: as many as its threads hold whole.
__host__ __device__ __forceinline__ int rows_of(int nb) { return kThreads / (4 * nb); }

struct Place {
    int64_t token;
    int head, j;      // j: first of the eight elements in the row
};

// False for the threads past the workgroup's last whole row.
__device__ __forceinline__ bool place(int heads, int nb, Place &p)
{
    const int per = 4 * nb, rows = rows_of(nb);
    const uint32_t row = small_quotient(threadIdx.x, 1.0f / (float)per);
    const int64_t row0 = block_of(blockIdx.y) * rows, token0 = quotient(row0, heads);
    const uint32_t h = (uint32_t)(row0 - token0 * heads) + row;   // below 65535 + 64
    const uint32_t more = small_quotient(h, 1.0f / (float)heads);
    p.token = token0 + more;
    p.head = (int)(h - more * (uint32_t)heads);
    p.j = ((int)threadIdx.x - (int)row * per) * 8;
    return row < (uint32_t)rows;
}

template <int kFmt, class T>
__global__ void __launch_bounds__(kThreads) mx_cache_write_kernel(MxCacheView c, const T *K, const T *V, int64_t k_tok,
                                                                  int64_t k_head, int64_t v_tok, int64_t v_head,
                                                                  int64_t tokens, const int64_t *slots)
{
    Place p;
    if (!place(c.heads, c.nb, p) || p.token >= tokens) return;
    const int64_t slot = slots[p.token];
    if (slot < 0 || slot >= c.n_pages * c.page) return;
    int64_t page;
    int at;
    find(c, slot, page, at);
    const Eight<T> ke = load_eight(K + p.token * k_tok + p.head * k_head + p.j, c.dim - p.j);
    const Eight<T> ve = load_eight(V + p.token * v_tok + p.head * v_head + p.j, c.dim - p.j);
    float k[8], v[8];
    ke.values(k);
    ve.values(v);
    const int64_t ph = page * c.heads + p.head, code = code_at<kFmt>(c, ph, at, p.j), scale = scale_at(c, ph, at, p.j);
    write8<kFmt>(k, c.k + code, c.ks + scale, p.j % kMxBlock == 0);
    write8<kFmt>(v, c.v + code, c.vs + scale, p.j % kMxBlock == 0);
}

template <int kFmt, class T>
__global__ void __launch_bounds__(kThreads) mx_cache_read_kernel(MxCacheView c, T *K, T *V, int64_t k_tok,
                                                                 int64_t k_head, int64_t v_tok, int64_t v_head,
                                                                 int64_t tokens, const int64_t *slots)
{
    Place p;
    if (!place(c.heads, c.nb, p) || p.token >= tokens || p.j >= c.dim) return;
    const int64_t slot = slots[p.token];
    float k[8] = {0, 0, 0, 0, 0, 0, 0, 0}, v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (slot >= 0 && slot < c.n_pages * c.page) {
        int64_t page;
        int at;
        find(c, slot, page, at);
        const int64_t ph = page * c.heads + p.head, code = code_at<kFmt>(c, ph, at, p.j),
                      scale = scale_at(c, ph, at, p.j);
        read8<kFmt>(c.k + code, c.ks + scale, k);
        read8<kFmt>(c.v + code, c.vs + scale, v);
    }
    store8<true>(K + p.token * k_tok + p.head * k_head + p.j, c.dim - p.j, k);
    store8<true>(V + p.token * v_tok + p.head * v_head + p.j, c.dim - p.j, v);
}

int64_t row_blocks(const MxCacheView &c, int64_t tokens)
{
    const int rows = rows_of(c.nb);
    return (tokens * c.heads + rows - 1) / rows;   // below 2^39 rows (host check)
}

}  // namespace

template <class T>
static hipError_t write_as(const MxCacheView &c, const MxRows &r, int64_t tokens, const int64_t *slots, dim3 grid,
                           hipStream_t s)
{
    auto kern = c.fmt == kFp4 ? mx_cache_write_kernel<kFp4, T> : mx_cache_write_kernel<kFp8, T>;
    hipLaunchKernelGGL(kern, grid, dim3(kThreads), 0, s, c, (const T *)r.K, (const T *)r.V, r.k_tok,
                       r.k_head, r.v_tok, r.v_head, tokens, slots);
    return hipGetLastError();
}

template <class T>
static hipError_t read_as(const MxCacheView &c, const MxRows &r, int64_t tokens, const int64_t *slots, dim3 grid,
                          hipStream_t s)
{
    auto kern = c.fmt == kFp4 ? mx_cache_read_kernel<kFp4, T> : mx_cache_read_kernel<kFp8, T>;
    hipLaunchKernelGGL(kern, grid, dim3(kThreads), 0, s, c, (T *)r.K, (T *)r.V, r.k_tok, r.k_head, r.v_tok,
                       r.v_head, tokens, slots);
    return hipGetLastError();
}

hipError_t launch_mx_cache_write(const MxCacheView &c, const MxRows &r, int64_t tokens, const int64_t *slots,
                                 hipStream_t s)
{
    const int64_t blocks = row_blocks(c, tokens);
    if (blocks <= 0) return hipSuccess;
    if (grid_rows(blocks) > 65535) return hipErrorInvalidValue;
    const dim3 grid(grid_x(blocks), (unsigned)grid_rows(blocks));
    LaunchTimer timer(s, "mx_cache_write_kernel");
    if (r.dtype == MPQ_F32) return write_as<float>(c, r, tokens, slots, grid, s);
    if (r.dtype == MPQ_F16) return write_as<_Float16>(c, r, tokens, slots, grid, s);
    return write_as<__bf16>(c, r, tokens, slots, grid, s);
}

hipError_t launch_mx_cache_read(const MxCacheView &c, const MxRows &r, int64_t tokens, const int64_t *slots,
                                hipStream_t s)
{
    const int64_t blocks = row_blocks(c, tokens);
    if (blocks <= 0) return hipSuccess;
    if (grid_rows(blocks) > 65535) return hipErrorInvalidValue;
    const dim3 grid(grid_x(blocks), (unsigned)grid_rows(blocks));
    LaunchTimer timer(s, "mx_cache_read_kernel");
    if (r.dtype == MPQ_F32) return read_as<float>(c, r, tokens, slots, grid, s);
    if (r.dtype == MPQ_F16) return read_as<_Float16>(c, r, tokens, slots, grid, s);
    return read_as<__bf16>(c, r, tokens, slots, grid, s);
}

}  // namespace mpq
