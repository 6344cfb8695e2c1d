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

// 32 bits from x = number of the element * 0x9E3779B1 + t * 0x3C6EF373 + seed: two rounds of xor-shift and multiplication (by the fractional
// parts of the golden ratio and of the roots of 5, 2 and 3).
__device__ __forceinline__ uint32_t counter_hash(uint32_t x)
{
    x = (x ^ (x >> 16)) * 0x6A09E667u;
    x = (x ^ (x >> 15)) * 0xBB67AE85u;
    return x ^ (x >> 16);
}

// 2^e for e in -127 .. 128 (2^128: 2^127, for an empty block)
__device__ __forceinline__ float two_to(int e) { return e >= -126 ? __builtin_bit_cast(float, (uint32_t)min(e + 127, 254) << 23) : 0x1p-127f; }

// The exponent of a block whose largest magnitude is `top`: -127 for an empty block.
__device__ __forceinline__ int block_exponent(float top)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, top);
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u);
    return top > 0.0f ? max(e, -126) : -127;
}

// x * 2^-e to an e4m3 code; `noise` in 0 .. 65535 decides between the neighbours; `least`: the smallest code that a nonzero x may get.
// y in units of its last kept bit (2^-9 below 2^-6) plus the noise's fraction, cut: a product by a power of two and one addition, as the
// definition has it.  An infinity or NaN becomes NaN.
__device__ __forceinline__ uint32_t encode(float x, float down, uint32_t noise, uint32_t least)
{
    const float y = fabsf(x) * down;
    const uint32_t exponent = max(__builtin_bit_cast(uint32_t, y) >> 23, 121u);
    uint32_t k = (uint32_t)__builtin_fmaf((float)noise, 0x1p-16f, __builtin_ldexpf(y, 130 - (int)exponent));
    if (least) k = max(k, x != 0.0f ? least : 0u);
    const uint32_t code = y < 0x1p9f ? (exponent << 3) + k - 121 * 8 : 0x7Fu;
    return code | (__builtin_bit_cast(uint32_t, x) >> 31) << 7;
}

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
    return v;
}

// The largest magnitude of a block, of those that are finite: an infinity is its own element's loss, and no scale for the others of its block (with its
// exponent they became 0, their u 2^111, whose square overflows in the next call: 256 parameters were NaN in the third).  Finite u are below
// 2^64, so e of a block of u is 56 at most, and the least code that its others get, 2^47, has a finite square.  (Infinities are sought where the
// maximum is one: 109 million elements 396.5 us, 399.9 with a look at every element and 394.3 with none.)
template <bool WHOLE>
__device__ __forceinline__ float block_top(const float (&x)[4], int n)
{
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; e++)
        if (WHOLE || e < n) top = fmaxf(top, fabsf(x[e]));
    top = wave_max(top);
    if (top == __builtin_inff()) {
        top = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const float a = fabsf(x[e]);
            if ((WHOLE || e < n) && a < __builtin_inff()) top = fmaxf(top, a);
        }
        top = wave_max(top);
    }
    return top;
}

template <typename T>
__device__ __forceinline__ float grad_of(T g);
template <>
__device__ __forceinline__ float grad_of(float g) { return g; }
template <>
__device__ __forceinline__ float grad_of(_Float16 g) { return (float)g; }
template <>
__device__ __forceinline__ float grad_of(__bf16 g) { return (float)g; }

template <typename T>
constexpr int type_of()
{
    return __is_same(T, float) ? FP6_F32 : (__is_same(T, __bf16) ? FP6_BF16 : FP6_F16);
}

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

// Four consecutive elements; WHOLE: all four exist, else `n` of them (the end of a tensor).
template <bool WHOLE, typename T, int W>
__device__ __forceinline__ void load4(const T* p, int n, T (&v)[W])
{
    typedef T vec __attribute__((ext_vector_type(4)));
    if (WHOLE) {
        const vec x = __builtin_nontemporal_load(reinterpret_cast<const vec*>(p));
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] = x[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] = e < n ? p[e] : T(0);
    }
}

template <bool WHOLE, typename T, int W>
__device__ __forceinline__ void store4(T* p, int n, const T (&v)[W])
{
    typedef T vec __attribute__((ext_vector_type(4)));
    if (WHOLE) {
        __builtin_nontemporal_store(vec{v[0], v[1], v[2], v[3]}, reinterpret_cast<vec*>(p));
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (e < n) p[e] = v[e];
    }
}

// What a lane holds of a block: four elements.
template <int BITS, typename G>
struct BlockIn {
    float p[4];
    G g[4];
    float m[4], v[4];        // 32 bits
    uint32_t cm, cv;         // 8 bits: four codes each, and the block's scale bytes
    uint32_t sm, sv;
};

template <int BITS, typename G, bool WHOLE>
__device__ __forceinline__ void load_block(const AdamwItem& it, int block, int lane, BlockIn<BITS, G>& in)
{
    const int at = block * 256 + 4 * lane, n = (int)it.count - at;
    load4<WHOLE>(it.param + at, n, in.p);
    load4<WHOLE>((const G*)it.grad + at, n, in.g);
    if (BITS == 32) {
        load4<WHOLE>((const float*)it.first + at, n, in.m);
        load4<WHOLE>((const float*)it.second + at, n, in.v);
    } else {
        const uint8_t *m = (const uint8_t*)it.first + at, *v = (const uint8_t*)it.second + at;
        if (WHOLE) {
            in.cm = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(m));
            in.cv = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(v));
        } else {
            in.cm = in.cv = 0;
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (e < n) {
                    in.cm |= (uint32_t)m[e] << (8 * e);
                    in.cv |= (uint32_t)v[e] << (8 * e);
                }
        }
        in.sm = it.first_scales[block];
        in.sv = it.second_scales[block];
    }
}

template <int BITS, typename G, typename C, bool WHOLE>
__device__ __forceinline__ void step_block(const AdamwItem& it, int block, int lane, const BlockIn<BITS, G>& in, const StepScalars& s)
{
#pragma clang fp contract(off)
    const int at = block * 256 + 4 * lane, n = (int)it.count - at;
    float p[4], m[4], v[4], u[4];
    if (BITS == 32) {
#pragma unroll
        for (int e = 0; e < 4; e++) {
            m[e] = in.m[e];
            v[e] = in.v[e];
        }
    } else {
        const float sm = two_to((int)in.sm - 127), sv = two_to((int)in.sv - 127);
        m[0] = __builtin_amdgcn_cvt_f32_fp8((int)in.cm, 0) * sm;
        m[1] = __builtin_amdgcn_cvt_f32_fp8((int)in.cm, 1) * sm;
        m[2] = __builtin_amdgcn_cvt_f32_fp8((int)in.cm, 2) * sm;
        m[3] = __builtin_amdgcn_cvt_f32_fp8((int)in.cm, 3) * sm;
        u[0] = __builtin_amdgcn_cvt_f32_fp8((int)in.cv, 0) * sv;
        u[1] = __builtin_amdgcn_cvt_f32_fp8((int)in.cv, 1) * sv;
        u[2] = __builtin_amdgcn_cvt_f32_fp8((int)in.cv, 2) * sv;
        u[3] = __builtin_amdgcn_cvt_f32_fp8((int)in.cv, 3) * sv;
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] = u[e] * u[e];
    }
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const float x = grad_of<G>(in.g[e]) * s.scale;
        m[e] = m[e] * s.b1 + x * s.c1;
        v[e] = v[e] * s.b2 + x * x * s.c2;
        u[e] = __builtin_sqrtf(v[e]);
        p[e] = in.p[e] * s.decay - m[e] / (u[e] * s.second + s.eps) * s.first;
    }
    store4<WHOLE>(it.param + at, n, p);
    if (sizeof(C) == 2) {
        C c[4];
#pragma unroll
        for (int e = 0; e < 4; e++) c[e] = (C)p[e];
        store4<WHOLE>((C*)it.copy + at, n, c);
    }
    if (BITS == 32) {
        store4<WHOLE>((float*)it.first + at, n, m);
        store4<WHOLE>((float*)it.second + at, n, v);
    } else {
        const int em = block_exponent(block_top<WHOLE>(m, n)), eu = block_exponent(block_top<WHOLE>(u, n));
        const float dm = two_to(-em), du = two_to(-eu);
        const uint32_t id = (it.id + (uint32_t)at) * 0x9E3779B1u + s.salt;
        uint32_t cm = 0, cu = 0;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const uint32_t noise = counter_hash(id + e * 0x9E3779B1u);
            cm |= encode(m[e], dm, noise >> 16, 0) << (8 * e);
            cu |= encode(u[e], du, noise & 0xFFFFu, 1) << (8 * e);
        }
        uint8_t *to_m = (uint8_t*)it.first + at, *to_u = (uint8_t*)it.second + at;
        if (WHOLE) {
            __builtin_nontemporal_store(cm, reinterpret_cast<uint32_t*>(to_m));
            __builtin_nontemporal_store(cu, reinterpret_cast<uint32_t*>(to_u));
        } else {
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (e < n) {
                    to_m[e] = (uint8_t)(cm >> (8 * e));
                    to_u[e] = (uint8_t)(cu >> (8 * e));
                }
        }
        if (lane == 0) {
            it.first_scales[block] = (uint8_t)(em + 127);
            it.second_scales[block] = (uint8_t)(eu + 127);
        }
    }
}

// A workgroup walks over the items of the plan; a wavefront takes the blocks of 256 elements wave, wave + 4, ... of an item, the next one's loads
// in flight while it works on one.  Whole blocks take no branch; the last one of a tensor may be short.  Bound by memory: 109 million
// elements with states in 8 bits 397 us for 1.96 GB, 4.9 TB/s (a large copy: 5.2), with 126 vector instructions an element beside it;
// 20 million with states in 32 bits 122 us, 4.9 TB/s; 0.6 million 6.8 us, of which a plan of one block takes 5.0.
template <int BITS, typename G, typename C>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwHeader* __restrict__ plan, const AdamwItem* __restrict__ list, int64_t items,
                                                    int32_t* __restrict__ step, AdamwCall call)
{
#pragma clang fp contract(off)
    StepScalars s;
    const uint32_t t = (uint32_t)*step + 1;
    if (call.found_inf && *call.found_inf != 0.0f) return;
    // (not a plan, one of another kind, or fewer items than the caller says: nothing beyond it is touched)
    if (plan->magic != kAdamwMagic || plan->kind != adamw_kind(BITS, type_of<G>(), sizeof(C) == 2 ? type_of<C>() : FP6_NO_COPY)) return;
    items = min(items, (int64_t)plan->items);
    s.scale = call.grad_scale ? *call.grad_scale : 1.0f;
    const double lr = call.lr_device ? (double)*call.lr_device : call.lr;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    s.decay = (float)(1.0 - lr * call.weight_decay);
    s.b1 = (float)call.beta1;
    s.c1 = (float)(1.0 - call.beta1);
    s.b2 = (float)call.beta2;
    s.c2 = (float)(1.0 - call.beta2);
    s.eps = (float)call.eps;
    s.salt = t * 0x3C6EF373u + call.seed;

    // The blocks of a wavefront one after another: `per` of each of its items.  The item after the next is asked for, the next block is in flight.
    const int64_t mine = items > blockIdx.x ? (items - 1 - blockIdx.x) / gridDim.x + 1 : 0;
    auto item_at = [&](int64_t k) { return list[blockIdx.x + min(k, mine - 1) * gridDim.x]; };
    const uint32_t group = blockIdx.x % kArrivalGroups, groups = min(gridDim.x, (uint32_t)kArrivalGroups);
    const uint32_t members = (gridDim.x - 1 - group) / kArrivalGroups + 1;
    uint32_t arrival = 0, root = 0;
    AdamwItem it{}, next{};
    BlockIn<BITS, G> in[2];
    if (mine > 0) {
        it = item_at(0);
        if (wave < (int)(it.count / 256)) load_block<BITS, G, true>(it, wave, lane, in[0]);
        next = item_at(1);
    }
    // (behind the first loads)
    s.first = (float)(lr / (1.0 - power(call.beta1, t)));
    s.second = (float)(1.0 / sqrt(1.0 - power(call.beta2, t)));
    // The step is read, and the workgroup says so; the last one to say it counts the step on.
    __syncthreads();                     // (every wavefront has its step)
    if (threadIdx.x == 0) {
        arrival = __hip_atomic_fetch_add(&plan->arrived[1 + group].count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1;
        if (arrival == members) {
            __hip_atomic_store(&plan->arrived[1 + group].count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            root = __hip_atomic_fetch_add(&plan->arrived[0].count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1;
        }
    }
    int turn = 0;
    for (int64_t k = 0; k < mine; k++) {
        const AdamwItem after = item_at(k + 2);
        const int whole = (int)(it.count / 256), blocks = (int)((it.count + 255) / 256);
        for (int block = wave; block < blocks || block == wave; block += 4) {
            const bool last = block + 4 >= blocks;
            const AdamwItem& from = last ? next : it;
            const int to = last ? wave : block + 4;
            const bool fetch = (!last || k + 1 < mine) && to < (int)(from.count / 256);
            if (turn == 0) {
                if (fetch) load_block<BITS, G, true>(from, to, lane, in[1]);
                if (block < whole) step_block<BITS, G, C, true>(it, block, lane, in[0], s);
            } else {
                if (fetch) load_block<BITS, G, true>(from, to, lane, in[0]);
                if (block < whole) step_block<BITS, G, C, true>(it, block, lane, in[1], s);
            }
            turn ^= 1;
            if (block >= whole && block < blocks) {
                BlockIn<BITS, G> tail;
                load_block<BITS, G, false>(it, block, lane, tail);
                step_block<BITS, G, C, false>(it, block, lane, tail, s);
            }
        }
        it = next;
        next = after;
    }
    if (root == groups) {
        __hip_atomic_store(&plan->arrived[0].count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(step, (int32_t)t, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

template <int BITS, typename G>
static void launch_grad_type(int copy_type, dim3 grid, AdamwHeader* plan, int64_t items, int32_t* step, const AdamwCall& call, hipStream_t stream)
{
    if (copy_type == FP6_F16) hipLaunchKernelGGL((adamw_kernel<BITS, G, _Float16>), grid, dim3(256), 0, stream, plan, (const AdamwItem*)(plan + 1), items, step, call);
    else if (copy_type == FP6_BF16) hipLaunchKernelGGL((adamw_kernel<BITS, G, __bf16>), grid, dim3(256), 0, stream, plan, (const AdamwItem*)(plan + 1), items, step, call);
    else hipLaunchKernelGGL((adamw_kernel<BITS, G, float>), grid, dim3(256), 0, stream, plan, (const AdamwItem*)(plan + 1), items, step, call);
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
