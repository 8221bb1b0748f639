// Product of fp4 rows, Y = X W^T + b (mpq_mx_product, mpq_mx_linear), on the
// matrix cores' scaled 4-bit instruction: v_mfma_scale_f32_16x16x128 takes,
// from lane l, the 32 elements of one block of row l % 16 (16 bytes) and that
// block's scale byte, so a block's scale costs nothing beside its product,
// and sums 128 products (four blocks, one for each l / 16) in fp32.  Rows of
// W are the instruction's rows, tokens its columns.
//
// The order of the sum is free as long as both operands share it: in a chunk
// of 512 elements, lanes of group g = l / 16 take the blocks 4g .. 4g + 3, one
// for each of four instructions.  A lane then reads 64 consecutive bytes of
// its row and one aligned word of four scales, whose bytes the instructions
// select themselves.
#include <algorithm>

#include "mpq.h"
#include "mx.hpp"

namespace mpq {

namespace {

constexpr int kChunkBlocks = 16;   // a chunk: 512 elements, 256 bytes of a row

// One lane's share of a chunk of a row: blocks 4g .. 4g + 3 and their scales.
// A row holds nb blocks, a multiple of four, so a lane's four are all there
// or none is (zeros then).
struct Share {
    u32x4 c[4];
    uint32_t s;
};

__device__ __forceinline__ Share load_share(const uint8_t *codes, const uint8_t *scales, int64_t row, int nb, int blk)
{
    Share v;
    if (blk < nb) {
        const u32x4 *p = (const u32x4 *)(codes + (row * nb + blk) * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) v.c[i] = p[i];
        v.s = *(const uint32_t *)(scales + row * nb + blk);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v.c[i] = u32x4{0, 0, 0, 0};
        v.s = 0;
    }
    return v;
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
// sums meet in LDS, added in wavefront order.
constexpr int kFewWaves = 8;

template <int kNT>
__global__ void __launch_bounds__(kFewWaves *kWave) mx_few_kernel(MxProduct p)
{
    __shared__ __align__(16) float part[kFewWaves][kNT][kWave * 4];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int r = lane % 16, g = lane / 16;
    const int64_t c0 = (int64_t)blockIdx.x * 16, t0 = (int64_t)blockIdx.y * 16 * kNT;
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
    for (int k = wave * kChunkBlocks; k < nb; k += kFewWaves * kChunkBlocks) {
        const Share a = load_share(p.wc, p.ws, wrow, nb, k + 4 * g);
        Share b[kNT];
#pragma unroll
        for (int t = 0; t < kNT; ++t) b[t] = load_share(p.xc, p.xs, xrow[t], nb, k + 4 * g);
#pragma unroll
        for (int t = 0; t < kNT; ++t) acc[t] = multiply_chunk(a, b[t], acc[t]);
    }
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

}  // namespace

hipError_t launch_mx_product(const MxProduct &p, hipStream_t s)
{
    if (p.n <= 0 || p.c <= 0) return hipSuccess;
    const int nt = p.n <= 16 ? 1 : p.n <= 32 ? 2 : 4;
    const int64_t gx = (p.c + 15) / 16, gy = (p.n + 16 * nt - 1) / (16 * nt);
    if (gx > 0x7fffffffLL || gy > 65535) return hipErrorInvalidValue;
    LaunchTimer timer(s, "mx_few_kernel");
    auto kern = nt == 1 ? mx_few_kernel<1> : nt == 2 ? mx_few_kernel<2> : mx_few_kernel<4>;
    hipLaunchKernelGGL(kern, dim3((unsigned)gx, (unsigned)gy), dim3(kFewWaves * kWave), 0, s, p);
    return hipGetLastError();
}

}  // namespace mpq
