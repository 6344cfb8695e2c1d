// The plan of an AdamW step as it lies in device memory, and what a call adds to it.
#pragma once

#include "fp6_internal.hpp"

namespace fp6 {

constexpr int kAdamwItem = 4096;         // elements of a tensor that a workgroup takes at a time
constexpr uint32_t kAdamwMagic = 0x41445731u;

// [header][tensors][first block of each tensor][items]
struct AdamwHeader {
    uint32_t magic, arrived;             // workgroups that have finished (zero whenever no call runs)
    uint32_t tensors, state_bits;
    uint64_t blocks_at, items_at;        // byte offsets
    uint64_t items;
    uint64_t pad[3];
};

struct AdamwItem {
    uint32_t tensor, part;
};

struct AdamwCall {
    double lr, beta1, beta2, eps, weight_decay;
    const float *lr_device, *grad_scale, *found_inf;
    uint32_t seed;
};

hipError_t launch_adamw(int state_bits, int grad_type, int copy_type, AdamwHeader* plan, int64_t items, int32_t* step, const AdamwCall& call,
                        hipStream_t stream);

}  // namespace fp6
