// What the host passes to the optimizer kernel: up to kAdamTensors tensors by value.
#pragma once

#include "common.h"

namespace sdgp {

constexpr int kAdamTensors = 52;   // a launch's arguments stay below 4 KB
constexpr int kAdamBlock = 256;    // elements that share a scale in an 8-bit state
constexpr int64_t kAdamLaunch = 1 << 22;   // blocks of a launch: its threads are counted in 32 bits

struct AdamTensor {
    void* p;
    const void* g;
    void *m, *v;
    float *m_scale, *v_scale;      // 8-bit states
    uint16_t* copy;                // bf16 copy of an fp32 parameter, or null
    int64_t n;
};

struct AdamArgs {
    AdamTensor t[kAdamTensors];
    uint32_t first[kAdamTensors + 1];   // first block of each tensor, counted in this launch
    int count;
    int64_t base;                       // blocks of the call in front of this launch
    const float* grad_scale;
    float b1, one_b1, b2, one_b2, decay, rate, root_bc2, eps;
    uint32_t mix;
};

int adamw_launch(const AdamArgs& a, int param_dt, int grad_dt, int state_bits, hipStream_t stream);

}  // namespace sdgp
