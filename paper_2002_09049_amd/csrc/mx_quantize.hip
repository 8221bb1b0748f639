// Rows to fp4 blocks and back (mpq_mx_quantize, mpq_mx_dequantize).
//
// Both stream, bound by memory: a thread holds eight consecutive elements, so
// the four lanes of a quad hold a block and its largest magnitude takes two DPP
// steps, and 16-bit values come and go as whole 16-byte vectors, lane by lane
// (16 elements a thread on the way back, its stores 32 bytes apart: 107 us where
// eight take 69).  A workgroup takes 2048 consecutive elements of the rows
// laid end to end (each row w elements, w a multiple of 128 at or above d),
// whatever their length; only its first element's row takes a division of
// large numbers.
//
// 4096 x 25088: fp32 to fp4 79 us, 5.9 TB/s of the 466 MB that it moves; back to
// bf16 44 us, 5.9 TB/s of 260 MB.  A large copy, half reads and half writes,
// reaches 5.2 TB/s; these mostly read or mostly write, and the codes, just
// written when they were timed, may still lie in the last-level cache.
#include "mpq.h"
#include "mx_quantize.hpp"

namespace mpq {

namespace {

constexpr int kThreads = kRowThreads, kElems = kRowElems;

template <class T>
__global__ void __launch_bounds__(kThreads) mx_quantize_kernel(const T *X, int64_t rows, int d, int64_t ld, int w,
                                                               uint8_t *codes, uint8_t *scales)
{
    quantize_eight(block_of(blockIdx.y), X, rows, d, ld, w, codes, scales);
}

template <class T>
__global__ void __launch_bounds__(kThreads) mx_dequantize_kernel(const uint8_t *codes, const uint8_t *scales,
                                                                 int64_t rows, int d, int w, T *Y, int64_t ld)
{
    int64_t row;
    int j;
    place_eight(block_of(blockIdx.y), w, row, j);
    if (row >= rows || j >= d) return;
    const uint32_t c[1] = {*(const uint32_t *)(codes + row * (w / 2) + j / 2)};
    float x[8];
    mx_values<kFp4>(c, scales[row * (w / kMxBlock) + j / kMxBlock], x);
    store8<true>(Y + row * ld + j, d - j, x);
}

template <class T>
hipError_t quantize_as(const T *X, int64_t rows, int d, int64_t ld, int w, uint8_t *codes, uint8_t *scales,
                       dim3 grid, hipStream_t s)
{
    hipLaunchKernelGGL(mx_quantize_kernel<T>, grid, dim3(kThreads), 0, s, X, rows, d, ld, w, codes, scales);
    return hipGetLastError();
}

template <class T>
hipError_t dequantize_as(const uint8_t *codes, const uint8_t *scales, int64_t rows, int d, int w, T *Y, int64_t ld,
                         dim3 grid, hipStream_t s)
{
    hipLaunchKernelGGL(mx_dequantize_kernel<T>, grid, dim3(kThreads), 0, s, codes, scales, rows, d, w, Y, ld);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_quantize(const void *X, int dtype, int64_t rows, int64_t d, int64_t ld, uint8_t *codes,
                              uint8_t *scales, hipStream_t s)
{
    const int w = (int)mx_row(d);
    const int64_t blocks = (rows * w + kElems - 1) / kElems;
    if (blocks <= 0) return hipSuccess;
    if (grid_rows(blocks) > 65535) return hipErrorInvalidValue;
    const dim3 grid(grid_x(blocks), (unsigned)grid_rows(blocks));
    LaunchTimer timer(s, "mx_quantize_kernel");
    if (dtype == MPQ_F32) return quantize_as((const float *)X, rows, (int)d, ld, w, codes, scales, grid, s);
    if (dtype == MPQ_F16) return quantize_as((const _Float16 *)X, rows, (int)d, ld, w, codes, scales, grid, s);
    return quantize_as((const __bf16 *)X, rows, (int)d, ld, w, codes, scales, grid, s);
}

hipError_t launch_mx_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t d, void *Y,
                                int dtype, int64_t ld, hipStream_t s)
{
    const int w = (int)mx_row(d);
    const int64_t blocks = (rows * w + kElems - 1) / kElems;
    if (blocks <= 0) return hipSuccess;
    if (grid_rows(blocks) > 65535) return hipErrorInvalidValue;
    const dim3 grid(grid_x(blocks), (unsigned)grid_rows(blocks));
    LaunchTimer timer(s, "mx_dequantize_kernel");
    if (dtype == MPQ_F32) return dequantize_as(codes, scales, rows, (int)d, w, (float *)Y, ld, grid, s);
    if (dtype == MPQ_F16) return dequantize_as(codes, scales, rows, (int)d, w, (_Float16 *)Y, ld, grid, s);
    return dequantize_as(codes, scales, rows, (int)d, w, (__bf16 *)Y, ld, grid, s);
}

}  // namespace mpq
