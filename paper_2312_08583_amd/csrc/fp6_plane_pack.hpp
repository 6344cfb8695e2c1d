// Rounding to the small formats and packing of a tile's planes (ZeroQuant(4+2) Section 4 Eq. 3, Section 5.1), shared by the quantizer and by
// the kernel that packs a weight a second time, turned.
#pragma once

#include "fp6_common.hpp"
#include "fp6_internal.hpp"

namespace fp6 {

// What dividing by one scale needs: the scale and minus its reciprocal, with the 2^12 of the bias shift (Section 5.2)
// folded in, so that quotients come out 2^-12 times the FP6 value.  A zero scale gives zero quotients.
struct Divisor {
    float s, neg_r;
};
__device__ __forceinline__ Divisor divisor_of(_Float16 S)
{
    const float s = (float)S * 4096.0f;
    return Divisor{s, s == 0.0f ? -0.0f : -1.0f / s};
}

// w / (S * 2^12), saturated at the format's largest magnitude: q0 = w * r is corrected by its exact remainder, two
// fused operations instead of the eight of an IEEE division.  Where the quotient is a midpoint of the code grid (few
// bits) the corrected quotient is that midpoint; any other quotient is at least 2^-17 (relative) away from every
// midpoint, far more than the 2^-24 that q can be off - so rounding q decides exactly as rounding the real quotient
// would.  The signs are arranged so that -0 stays -0: the remainder of an exact quotient is +0 and -r < 0.
template <int FMT>
__device__ __forceinline__ float quotient(float w, Divisor d)
{
    constexpr float kMax = (FMT == kE3M1 ? 24.0f : 28.0f) / 4096.0f;
    const float q0 = w * -d.neg_r;
    const float rem = __builtin_fmaf(d.s, q0, -w);
    return __builtin_amdgcn_fmed3f(__builtin_fmaf(rem, d.neg_r, q0), -kMax, kMax);
}

// E3M1: the quotient rounded to one mantissa bit (to nearest even) while it is still fp32; the conversion below is then
// exact.  From 2^-14 up (0.25 before the shift) half a unit minus one, plus the last kept bit, is added below the kept
// bits (a carry runs into the exponent as it should); below, the values are multiples of 2^-15, the spacing of fp32
// numbers around 384.
__device__ __forceinline__ float round_e3m1(float q)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, q);
    const uint32_t normal = (b + 0x1FFFFFu + ((b >> 22) & 1u)) & 0xFFC00000u;
    const float sub = __builtin_copysignf((fabsf(q) + 384.0f) - 384.0f, q);
    return fabsf(q) < 0x1p-14f ? sub : __builtin_bit_cast(float, normal);
}

__device__ __forceinline__ float low_half(uint32_t d) { return (float)__builtin_bit_cast(_Float16, (uint16_t)d); }
__device__ __forceinline__ float high_half(uint32_t d) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(d >> 16)); }

// Four weights to the bytes  s 0 0 e e e m m : the E5M2 number nearest to w / (S * 2^12) (to nearest even).  With the
// 2^12 taken out, E3M2's values are exactly E5M2's up to 28 * 2^-12, subnormals included (Eq. 5 read in eight bits), so
// the hardware conversion to E5M2 is the quantizer's rounding.  The bytes hold, in order, the weights a, b, c, d.
template <int FMT>
__device__ __forceinline__ uint32_t code_bytes(float a, float b, float c, float d, Divisor dv)
{
    float q[4] = {quotient<FMT>(a, dv), quotient<FMT>(b, dv), quotient<FMT>(c, dv), quotient<FMT>(d, dv)};
    if (FMT == kE3M1) {
#pragma unroll
        for (int e = 0; e < 4; e++) q[e] = round_e3m1(q[e]);
    }
    int u = __builtin_amdgcn_cvt_pk_bf8_f32(q[0], q[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(q[2], q[3], u, true);
}

// One lane slot of one tile (64 weights): v[f] = the eight consecutive weights of fragment f = 2t + q, i.e. of channel
// 16t + i at k block q; d[t] = the channel's divisor.  Writes the slot's 32 + 16 (FP5: 8) bytes of the two planes.
template <int FMT>
__device__ __forceinline__ void pack_slot(const u32x4 (&v)[8], const Divisor (&d)[4], u32x4* __restrict__ hi,
                                          u32x4* __restrict__ lo, size_t tile, int slot)
{
    uint32_t hiw[8], low[4] = {0, 0, 0, 0};
    if (FMT == kE3M2H) {
#pragma unroll
        for (int q = 0; q < 2; q++) {
            // the unit's codes as a string of 192 bits, 48 per fragment
            uint32_t T[6], head[4], tail[4];
#pragma unroll
            for (int t = 0; t < 4; t++) {
                const u32x4 w = v[2 * t + q];
                uint32_t x[2];
#pragma unroll
                for (int p = 0; p < 2; p++) {
                    const uint32_t u = code_bytes<FMT>(low_half(w[2 * p]), high_half(w[2 * p]), low_half(w[2 * p + 1]),
                                                       high_half(w[2 * p + 1]), d[t]);
                    const uint32_t c = ((u >> 2) & 0x20202020u) | (u & 0x1F1F1F1Fu);          // four codes, a byte each
                    const uint32_t y = (c & 0x003F003Fu) | ((c & 0x3F003F00u) >> 2);          // two pairs of 12 bits
                    x[p] = (y & 0xFFFu) | ((y >> 4) & 0xFFF000u);                             // 24 bits
                }
                head[t] = x[0] | (x[1] << 24);
                tail[t] = x[1] >> 8;
            }
            T[0] = head[0];
            T[1] = tail[0] | (head[1] << 16);
            T[2] = (head[1] >> 16) | (tail[1] << 16);
            T[3] = head[2];
            T[4] = tail[2] | (head[3] << 16);
            T[5] = (head[3] >> 16) | (tail[3] << 16);
            // split the string by kind of bit (the inverse of merge_unit)
            low[2 * q] = (T[0] & ~kSE0) | (T[1] & ~kSE1) | (T[2] & ~kSE2);
            low[2 * q + 1] = (T[3] & ~kSE0) | (T[4] & ~kSE1) | (T[5] & ~kSE2);
            hiw[4 * q + 0] = (T[0] & kSE0) | (T[4] & ~kSE0);
            hiw[4 * q + 1] = (T[1] & kSE1) | ((T[4] & 0x0C30C30Cu) << 2);
            hiw[4 * q + 2] = (T[2] & kSE2) | ((T[5] & 0x030C30C3u) << 2);
            const uint32_t r5 = T[5] & kFromA3;
            hiw[4 * q + 3] = (T[3] & kSE0) | (r5 << 2) | (r5 >> 30);
        }
    } else {
#pragma unroll
        for (int f = 0; f < 8; f++) {
            // bytes 0..3 of a plane dword carry elements 0, 2, 1, 3 of their group of four
            uint32_t u[2];
#pragma unroll
            for (int p = 0; p < 2; p++)
                u[p] = code_bytes<FMT>(low_half(v[f][2 * p]), low_half(v[f][2 * p + 1]), high_half(v[f][2 * p]),
                                       high_half(v[f][2 * p + 1]), d[f >> 1]);
            hiw[f] = (u[0] & 0x1C1C1C1Cu) | ((u[1] & 0x1C1C1C1Cu) << 3) | ((u[0] >> 7) & 0x01010101u) |
                     ((u[1] >> 6) & 0x02020202u);
            if (FMT == kE3M2)
                low[f >> 1] |= ((u[0] & 0x03030303u) | ((u[1] & 0x03030303u) << 2)) << (4 * (f & 1));
            else
                low[f >> 2] |= (((u[0] >> 1) & 0x01010101u) | (u[1] & 0x02020202u)) << (2 * (f & 3));
        }
    }
    u32x4* hp = hi + tile * kHiTileVec + slot;
    hp[0] = u32x4{hiw[0], hiw[1], hiw[2], hiw[3]};
    hp[64] = u32x4{hiw[4], hiw[5], hiw[6], hiw[7]};
    if (FMT != kE3M1) lo[tile * kLoTileVec + slot] = u32x4{low[0], low[1], low[2], low[3]};
    else reinterpret_cast<u32x2*>(lo)[tile * 64 + slot] = u32x2{low[0], low[1]};
}

}  // namespace fp6
