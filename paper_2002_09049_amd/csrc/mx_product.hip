// Product of fp4 rows, Y = X W^T + b (mpq_mx_product, mpq_mx_linear): the
// kernels over the whole of W, and which one a call takes.
#include <algorithm>
#include <cmath>

#include "mx_product.hpp"

namespace mpq {

namespace {

template <int kNT>
__global__ void __launch_bounds__(kFewWaves *kWave) mx_few_kernel(MxProduct p)
{
    const int64_t c0 = block_of(blockIdx.z) * 16, t0 = (int64_t)blockIdx.y * 16 * kNT;
    if (c0 >= p.c) return;
    few_product<kNT, kFewWaves>(p, c0, t0, [](int64_t token) { return token; });
}

template <int kN, class T>
__global__ void __launch_bounds__(kFewWaves *kWave) mx_token_kernel(MxProduct p, const T *X, int64_t x_ld, int d)
{
    const int64_t c0 = block_of(blockIdx.z) * 16;
    if (c0 >= p.c) return;
    token_product<kN, kFewWaves, T>(p, c0, 0, (int)p.n, d, [=](int64_t token) { return X + token * x_ld; },
                         [](int) { return false; });
}

template <int kTM, int kTN>
__global__ void __launch_bounds__(256) mx_tile_kernel(MxProduct p)
{
    constexpr int kBM = 64 * kTM, kBN = 64 * kTN;
    int tm, tn;
    if (!tile_of((int)((p.c + kBM - 1) / kBM), (int)((p.n + kBN - 1) / kBN), tm, tn)) return;
    tile_product<kTM, kTN, false>(p, (int64_t)tm * kBM, (int64_t)tn * kBN, MxGather{});
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
