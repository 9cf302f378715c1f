// What the host passes to the optimizer kernel: up to kAdamTensors tensors by value.
#pragma once

#include "common.h"

namespace sdgp {

constexpr int kAdamTensors = 48;                      // a launch's arguments stay below 4 KB
constexpr int kAdamBlock = 256;                       // elements that share a scale in an 8-bit state
constexpr int kAdamTile = 16;                         // blocks of a workgroup
constexpr int64_t kAdamLaunch = (int64_t)1 << 22;     // tiles of a launch: its threads are counted in 32 bits

struct AdamTensor {
    void* p;
    const void* g;
    void *m, *v;
    float *m_scale, *v_scale;      // 8-bit states
    uint16_t* copy;                // bf16 copy of an fp32 parameter, or null
    int64_t n;
    int64_t block;                 // its first block, counted in the call
};

struct AdamArgs {
    AdamTensor t[kAdamTensors];
    uint32_t first[kAdamTensors + 1];   // first tile of each tensor, counted in the launch
    int count;
    uint32_t mix;
    const float* grad_scale;
    // what the formula takes, computed in 64 bits
    float b1, one_b1, b2, one_b2, decay, rate, inv_root_bc2, eps;
};
static_assert(sizeof(AdamArgs) <= 4096, "a launch's arguments");

int adamw_launch(const AdamArgs& a, int param_dt, int grad_dt, int state_bits, hipStream_t stream);

}  // namespace sdgp
