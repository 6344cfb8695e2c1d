// One AdamW step over many tensors at once, for gfx950.
//
//   g' = scale * g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,  u = sqrt(v)
//   p = p (1 - lr wd) - lr / (1 - b1^t) * m / (u / sqrt(1 - b2^t) + eps)
// Every operation is fp32, rounded once, in this order (no contraction): the step is a function of its inputs, bit for bit.
//
// States in 8 bits: m and u as e4m3 numbers times one power of two per 256 elements, the smallest that brings the block's largest
// magnitude to 448 or below.  (u, not v: the root halves the range in binades, and 2^-9 .. 448 then spans eleven decades of v.)  The last
// kept bit is rounded up or down by 16 bits of a counter hash: a second moment changes by a thousandth a step, and rounding to
// nearest, in steps of an eighth, would never let it move.  A u that is not zero does not become zero: the next step divides by it.
#include "fp6_adamw.hpp"

#include "fp6_common.hpp"

namespace fp6 {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

// 32 bits from the number of an element, the step and the seed: two rounds of xor-shift and multiplication (by the fractional
// parts of the golden ratio and of the roots of 5, 2 and 3).
__device__ __forceinline__ uint32_t counter_hash(uint32_t id, uint32_t salt)
{
    uint32_t x = id * 0x9E3779B1u + salt;
    x = (x ^ (x >> 16)) * 0x6A09E667u;
    x = (x ^ (x >> 15)) * 0xBB67AE85u;
    return x ^ (x >> 16);
}

__device__ __forceinline__ float two_to(int e) { return e >= -126 ? __builtin_bit_cast(float, (uint32_t)(e + 127) << 23) : 0x1p-127f; }

// The exponent of a block whose largest magnitude is `top`: -127 for an empty block.
__device__ __forceinline__ int block_exponent(float top)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, top);
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u);
    return top > 0.0f ? max(e, -126) : -127;
}

// x * 2^-e to an e4m3 code; `noise` in 0 .. 65535 decides between the neighbours; `least`: the smallest code that a nonzero x may get.
__device__ __forceinline__ uint32_t encode(float x, float down, uint32_t noise, int least)
{
    const float y = fabsf(x) * down;
    const int ey = max((int)(__builtin_bit_cast(uint32_t, y) >> 23) - 127, -6);
    int k = (int)floorf(y * two_to(3 - ey) + (float)noise * 0x1p-16f);
    if (x != 0.0f) k = max(k, least);
    const uint32_t code = y < 0x1p9f ? (uint32_t)(((ey + 6) << 3) + k) : 0x7Fu;          // an infinity or NaN: NaN
    return code | (__builtin_bit_cast(uint32_t, x) >> 31) << 7;
}

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
    return v;
}

template <typename T>
__device__ __forceinline__ float grad_of(T g);
template <>
__device__ __forceinline__ float grad_of(float g) { return g; }
template <>
__device__ __forceinline__ float grad_of(_Float16 g) { return (float)g; }
template <>
__device__ __forceinline__ float grad_of(__bf16 g) { return (float)g; }

struct StepScalars {
    float decay, first, second, b1, c1, b2, c2, eps, scale;
    uint32_t salt;
};

// b^t by squaring, in double
__device__ __forceinline__ double power(double b, uint32_t t)
{
    double r = 1.0;
    for (; t; t >>= 1, b *= b)
        if (t & 1) r *= b;
    return r;
}

// Four consecutive elements of a block of 256: `n` of them exist (the last block of a tensor may be short).
template <typename T, int W>
__device__ __forceinline__ void load4(const T* p, int n, T (&v)[W])
{
    typedef T vec __attribute__((ext_vector_type(4)));
    if (n >= 4) {
        const vec x = *reinterpret_cast<const vec*>(p);
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] = x[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] = e < n ? p[e] : T(0);
    }
}

template <typename T, int W>
__device__ __forceinline__ void store4(T* p, int n, const T (&v)[W])
{
    typedef T vec __attribute__((ext_vector_type(4)));
    if (n >= 4) {
        *reinterpret_cast<vec*>(p) = vec{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (e < n) p[e] = v[e];
    }
}

// A workgroup walks over the items of the plan: 4096 elements of a tensor, four blocks of 256 for each of its wavefronts.
template <int BITS, typename G, typename C>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwHeader* __restrict__ plan, int64_t items, int32_t* __restrict__ step, AdamwCall call)
{
#pragma clang fp contract(off)
    if (call.found_inf && *call.found_inf != 0.0f) return;
    const uint32_t t = (uint32_t)*step + 1;
    const double lr = call.lr_device ? (double)*call.lr_device : call.lr;
    StepScalars s;
    s.decay = (float)(1.0 - lr * call.weight_decay);
    s.first = (float)(lr / (1.0 - power(call.beta1, t)));
    s.second = (float)(1.0 / sqrt(1.0 - power(call.beta2, t)));
    s.b1 = (float)call.beta1;
    s.c1 = (float)(1.0 - call.beta1);
    s.b2 = (float)call.beta2;
    s.c2 = (float)(1.0 - call.beta2);
    s.eps = (float)call.eps;
    s.scale = call.grad_scale ? *call.grad_scale : 1.0f;
    s.salt = t * 0x3C6EF373u + call.seed;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const AdamwItem* list = reinterpret_cast<const AdamwItem*>(reinterpret_cast<const unsigned char*>(plan) + plan->items_at);
    const fp6_adamw_tensor* tensors = reinterpret_cast<const fp6_adamw_tensor*>(plan + 1);
    const uint32_t* first_block = reinterpret_cast<const uint32_t*>(reinterpret_cast<const unsigned char*>(plan) + plan->blocks_at);
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const AdamwItem it = list[item];
        const fp6_adamw_tensor T = tensors[it.tensor];
        const uint32_t id0 = first_block[it.tensor] * 256u;
        const int64_t base = (int64_t)it.part * kAdamwItem + wave * (kAdamwItem / 4);
#pragma unroll 2
        for (int b = 0; b < kAdamwItem / 1024; b++) {
            const int64_t block = base + b * 256;
            if (block >= T.count) break;
            const int64_t at = block + 4 * lane, left = T.count - at;
            const int n = left >= 4 ? 4 : (left > 0 ? (int)left : 0);
            float p[4], m[4], v[4], u[4];
            G g[4];
            load4(T.param + at, n, p);
            load4((const G*)T.grad + at, n, g);
            if (BITS == 32) {
                load4((const float*)T.first + at, n, m);
                load4((const float*)T.second + at, n, v);
            } else {
                uint8_t cm[4], cv[4];
                load4((const uint8_t*)T.first + at, n, cm);
                load4((const uint8_t*)T.second + at, n, cv);
                const float sm = two_to((int)T.first_scales[block >> 8] - 127), sv = two_to((int)T.second_scales[block >> 8] - 127);
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    m[e] = __builtin_amdgcn_cvt_f32_fp8((int)cm[e], 0) * sm;
                    const float r = __builtin_amdgcn_cvt_f32_fp8((int)cv[e], 0) * sv;
                    v[e] = r * r;
                }
            }
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float x = grad_of<G>(g[e]) * s.scale;
                m[e] = m[e] * s.b1 + x * s.c1;
                v[e] = v[e] * s.b2 + x * x * s.c2;
                u[e] = __builtin_sqrtf(v[e]);
                p[e] = p[e] * s.decay - m[e] / (u[e] * s.second + s.eps) * s.first;
            }
            store4(T.param + at, n, p);
            if (sizeof(C) == 2) {
                C c[4];
#pragma unroll
                for (int e = 0; e < 4; e++) c[e] = (C)p[e];
                store4((C*)T.copy + at, n, c);
            }
            if (BITS == 32) {
                store4((float*)T.first + at, n, m);
                store4((float*)T.second + at, n, v);
            } else {
                float tm = 0.0f, tu = 0.0f;
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (e < n) {
                        tm = fmaxf(tm, fabsf(m[e]));
                        tu = fmaxf(tu, u[e]);
                    }
                const int em = block_exponent(wave_max(tm)), eu = block_exponent(wave_max(tu));
                const float dm = em == -127 ? 0x1p127f : two_to(-em), du = eu == -127 ? 0x1p127f : two_to(-eu);
                uint8_t cm[4], cu[4];
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const uint32_t noise = counter_hash(id0 + (uint32_t)at + e, s.salt);
                    cm[e] = (uint8_t)encode(m[e], dm, noise >> 16, 0);
                    cu[e] = (uint8_t)encode(u[e], du, noise & 0xFFFFu, 1);
                }
                store4((uint8_t*)T.first + at, n, cm);
                store4((uint8_t*)T.second + at, n, cu);
                if (lane == 0) {
                    T.first_scales[block >> 8] = (uint8_t)(em + 127);
                    T.second_scales[block >> 8] = (uint8_t)(eu + 127);
                }
            }
        }
    }
    // Every workgroup has read the step before it arrives here; the last one counts it on.
    __syncthreads();
    if (threadIdx.x == 0) {
        const uint32_t old = __hip_atomic_fetch_add(&plan->arrived, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
        if (old == gridDim.x - 1) {
            __hip_atomic_store(&plan->arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            *step = (int32_t)t;
        }
    }
}

template <int BITS, typename G>
static void launch_grad_type(int copy_type, dim3 grid, AdamwHeader* plan, int64_t items, int32_t* step, const AdamwCall& call, hipStream_t stream)
{
    if (copy_type == FP6_F16) hipLaunchKernelGGL((adamw_kernel<BITS, G, _Float16>), grid, dim3(256), 0, stream, plan, items, step, call);
    else if (copy_type == FP6_BF16) hipLaunchKernelGGL((adamw_kernel<BITS, G, __bf16>), grid, dim3(256), 0, stream, plan, items, step, call);
    else hipLaunchKernelGGL((adamw_kernel<BITS, G, float>), grid, dim3(256), 0, stream, plan, items, step, call);
}

template <int BITS>
static void launch_bits(int grad_type, int copy_type, dim3 grid, AdamwHeader* plan, int64_t items, int32_t* step, const AdamwCall& call, hipStream_t stream)
{
    if (grad_type == FP6_F16) launch_grad_type<BITS, _Float16>(copy_type, grid, plan, items, step, call, stream);
    else if (grad_type == FP6_BF16) launch_grad_type<BITS, __bf16>(copy_type, grid, plan, items, step, call, stream);
    else launch_grad_type<BITS, float>(copy_type, grid, plan, items, step, call, stream);
}

hipError_t launch_adamw(int state_bits, int grad_type, int copy_type, AdamwHeader* plan, int64_t items, int32_t* step, const AdamwCall& call,
                        hipStream_t stream)
{
    // eight workgroups of four wavefronts fill a compute unit
    const dim3 grid((unsigned)(items < 1 ? 1 : (items < 2048 ? items : 2048)));
    if (state_bits == 8) launch_bits<8>(grad_type, copy_type, grid, plan, items, step, call, stream);
    else launch_bits<32>(grad_type, copy_type, grid, plan, items, step, call, stream);
    return hipGetLastError();
}

}  // namespace fp6
