// The gradient of a frozen layer by its input, for gfx950: dX = dY W with W[n][k] = S_n c[n][k] held in codes.
//
// The sum runs over the output channels n, and the planes are laid out for sums over k.  So the weight is packed a second time, turned
// (offline, from the planes: 0.75 byte a weight more), and the layer's own kernels compute the sum: they take [K, N] codes for a
// layer that has N inputs and K outputs.  The row scale S_n multiplies terms of that sum, not its result; it goes into dY as
// rho_n = S_n / 2^E with 2^E the power of two at or above the largest scale, and 2^E is the scale of every output.
#include "fp6_plane_pack.hpp"

namespace fp6 {

// ratio[n] = S_n / 2^E (exact), scales_t[k] = 2^E.  One workgroup; the largest scale is found on the bit patterns.
__global__ __launch_bounds__(1024) void turned_scales_kernel(const uint16_t* __restrict__ scales, int64_t N, int64_t K,
                                                             uint16_t* __restrict__ scales_t, float* __restrict__ ratio)
{
    __shared__ uint32_t top;
    if (threadIdx.x == 0) top = 0;
    __syncthreads();
    uint32_t mx = 0;
    for (int64_t n = threadIdx.x; n < N; n += 1024) mx = max(mx, (uint32_t)scales[n] & 0x7FFFu);
    atomicMax(&top, mx);
    __syncthreads();
    // S <= 2^e <= 2^15 (scales of finite weights are below 2341; larger ones give ratios up to 2)
    const uint32_t b = __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(_Float16, (uint16_t)top));
    const int e = top == 0 ? 0 : min((int)(b >> 23) - 127 + ((b & 0x7FFFFFu) != 0), 15);
    const float power = __builtin_bit_cast(float, (uint32_t)(127 + e) << 23), inverse = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
    for (int64_t n = threadIdx.x; n < N; n += 1024) ratio[n] = (float)__builtin_bit_cast(_Float16, scales[n]) * inverse;
    for (int64_t k = threadIdx.x; k < K; k += 1024) scales_t[k] = __builtin_bit_cast(uint16_t, (_Float16)power);
}

// Planes of [N, K] to planes of [K, N].  A wavefront takes a tile: its codes as numbers (exact in fp16) go to LDS by rows of n, and
// come back as the eight consecutive n of a channel k that a slot of the turned tile holds.
template <int FMT>
__global__ __launch_bounds__(256) void turn_planes_kernel(const u32x4* __restrict__ hi, const u32x4* __restrict__ lo, int64_t N, int64_t K,
                                                          u32x4* __restrict__ hi_t, u32x4* __restrict__ lo_t)
{
    constexpr int kLd = kTile + 2;
    __shared__ uint16_t value[4][kTile * kLd];
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const uint32_t ktiles = (uint32_t)(K / kTile), ntiles = (uint32_t)(N / kTile), tile = blockIdx.x * 4 + wave;
    if (tile >= ntiles * ktiles) return;
    uint16_t* own = value[wave];
    const TileRaw r = load_tile<FMT>(hi, lo, tile, lane);
#pragma unroll
    for (int q = 0; q < 2; q++) {
        half8 w[4];
        unpack_kblock<kHalfMul, FMT>(r, q, w);
#pragma unroll
        for (int t = 0; t < 4; t++) {
            // (five bits: the padded operand, which the multiplication by 2^12 turns into the value)
            const half8 v = FMT == kE3M1 ? w[t] * (_Float16)4096.0f : w[t];
#pragma unroll
            for (int e = 0; e < 8; e++) own[(16 * t + i) * kLd + 32 * q + 8 * g + e] = __builtin_bit_cast(uint16_t, (_Float16)v[e]);
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    u32x4 v[8];
#pragma unroll
    for (int f = 0; f < 8; f++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const uint32_t k = 16 * (f >> 1) + i, n = 32 * (f & 1) + 8 * g + 2 * e;
            v[f][e] = own[n * kLd + k] | (uint32_t)own[(n + 1) * kLd + k] << 16;
        }
    const Divisor one = divisor_of((_Float16)1.0f);
    const Divisor d[4] = {one, one, one, one};
    pack_slot<FMT>(v, d, hi_t, lo_t, (size_t)(tile % ktiles) * ntiles + tile / ktiles, lane);
}

// out = dY * ratio, rounded to the type of dY: the one rounding that the gradient has beside that of its result (with the scale inside the
// sum a product of 11 + 11 bits has to become an operand of 11, or 8, bits on one side or the other).  In fp16 that holds down to 2^-14: the small products of
// small gradients, or of channels far below the largest scale, lose bits as fp16 numbers of their size do.  Rows lifted by a power of two for the product and lowered
// after it keep them, for a launch more in every call (16 x 4096 x 4096 13.0 us for 9.0): left to the caller's loss scale.
// A thread keeps the ratios of its eight columns and walks down the rows: 2048 x 22016 30 us for 180 MB, 5.9 TB/s; a few rows 2.3 us, a launch.
template <bool BF16>
__global__ __launch_bounds__(256) void scale_rows_kernel(const u32x4* __restrict__ dY, const float4v* __restrict__ ratio, int64_t M,
                                                         int64_t per_row, u32x4* __restrict__ out)
{
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= per_row) return;
    const float4v a = ratio[2 * c], b = ratio[2 * c + 1];
#pragma unroll 4
    for (int64_t row = blockIdx.y; row < M; row += gridDim.y) {
        const u32x4 d = dY[row * per_row + c];
        u32x4 y;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const float s0 = e < 2 ? a[2 * (e & 1)] : b[2 * (e & 1)], s1 = e < 2 ? a[2 * (e & 1) + 1] : b[2 * (e & 1) + 1];
            if (BF16) {
                const float x0 = __builtin_bit_cast(float, d[e] << 16) * s0, x1 = __builtin_bit_cast(float, d[e] & 0xFFFF0000u) * s1;
                y[e] = __builtin_bit_cast(uint16_t, (__bf16)x0) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x1) << 16;
            } else {
                const float x0 = low_half(d[e]) * s0, x1 = high_half(d[e]) * s1;
                y[e] = __builtin_bit_cast(uint16_t, (_Float16)x0) | (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x1) << 16;
            }
        }
        out[row * per_row + c] = y;
    }
}

hipError_t launch_transpose_pack(int format, const void* hi, const void* lo, const uint16_t* scales, int64_t N, int64_t K, void* hi_t,
                                 void* lo_t, uint16_t* scales_t, float* ratio, hipStream_t stream)
{
    hipLaunchKernelGGL(turned_scales_kernel, dim3(1), dim3(1024), 0, stream, scales, N, K, scales_t, ratio);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)(((N / kTile) * (K / kTile) + 3) / 4));
    const u32x4 *h = (const u32x4*)hi, *l = (const u32x4*)lo;
    if (format == kE3M2) hipLaunchKernelGGL(turn_planes_kernel<kE3M2>, grid, dim3(256), 0, stream, h, l, N, K, (u32x4*)hi_t, (u32x4*)lo_t);
    else if (format == kE3M1) hipLaunchKernelGGL(turn_planes_kernel<kE3M1>, grid, dim3(256), 0, stream, h, l, N, K, (u32x4*)hi_t, (u32x4*)lo_t);
    else hipLaunchKernelGGL(turn_planes_kernel<kE3M2H>, grid, dim3(256), 0, stream, h, l, N, K, (u32x4*)hi_t, (u32x4*)lo_t);
    return hipGetLastError();
}

hipError_t launch_scale_rows(bool bf16, const uint16_t* dY, const float* ratio, int64_t M, int64_t N, uint16_t* out, hipStream_t stream)
{
    // about 2048 workgroups, each at least one row
    const int64_t per_row = N / 8, across = (per_row + 255) / 256, down = (2047 + across) / across;
    const dim3 grid((unsigned)across, (unsigned)(M < down ? M : down));
    if (bf16) hipLaunchKernelGGL(scale_rows_kernel<true>, grid, dim3(256), 0, stream, (const u32x4*)dY, (const float4v*)ratio, M, per_row, (u32x4*)out);
    else hipLaunchKernelGGL(scale_rows_kernel<false>, grid, dim3(256), 0, stream, (const u32x4*)dY, (const float4v*)ratio, M, per_row, (u32x4*)out);
    return hipGetLastError();
}

}  // namespace fp6
