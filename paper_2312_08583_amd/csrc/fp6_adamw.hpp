// The plan of an AdamW step as it lies in device memory, and what a call adds to it.
#pragma once

#include "fp6_internal.hpp"

namespace fp6 {

constexpr uint32_t kAdamwMagic = 0x41445732u;

// Elements of a tensor that a workgroup takes at a time: each of its four wavefronts one block of 256, or four.  Few elements are
// spread over more workgroups (0.6 million: 612 items of 1024, where 4096 left three compute units in eight idle).
constexpr int64_t adamw_item(int64_t elements) { return elements <= (int64_t)4 << 20 ? 1024 : 4096; }

// Workgroups that have read the step are counted in two stages, 64 counters on lines of their own and one for those: additions to one
// address follow one another at 13 ns, and 2048 of them alone took 27 us.
constexpr int kArrivalGroups = 64;

// What the addresses of a plan were worked out with: a call of another kind would read and write beside its tensors.
constexpr uint32_t adamw_kind(int state_bits, int grad_type, int copy_type)
{
    return (uint32_t)state_bits | (uint32_t)grad_type << 8 | (uint32_t)(copy_type & 0xFF) << 16;
}

// [header][items]
struct AdamwHeader {
    uint32_t magic, kind;
    uint64_t items;
    uint32_t unused[28];
    struct {
        uint32_t count, unused[31];
    } arrived[kArrivalGroups + 1];       // zero whenever no call runs
};

// One item, all that a workgroup reads before the tensors themselves: its pointers, the number of its first element (for the hash) and how many.
struct AdamwItem {
    float* param;
    const void* grad;
    void *first, *second;
    uint8_t *first_scales, *second_scales;
    uint16_t* copy;
    uint32_t id, count;
};
static_assert(sizeof(AdamwHeader) == 128 * (kArrivalGroups + 2) && sizeof(AdamwItem) == 64, "the plan is lines of 128 bytes");

struct AdamwCall {
    double lr, beta1, beta2, eps, weight_decay;
    const float *lr_device, *grad_scale, *found_inf;
    uint32_t seed;
};

hipError_t launch_adamw(int state_bits, int grad_type, int copy_type, AdamwHeader* plan, int64_t items, int32_t* step, const AdamwCall& call,
                        hipStream_t stream);

}  // namespace fp6
