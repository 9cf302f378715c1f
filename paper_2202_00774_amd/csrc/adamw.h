// What the host passes to the optimizer kernel: up to kAdamTensors tensors by value.
#pragma once

#include "common.h"

namespace sdgp {

constexpr int kAdamBlock = 256;                       // elements that share a scale in an 8-bit state
// Blocks of a workgroup: four wavefronts with four each in flight for fp32 states, one each for 8-bit ones, where a block's
// arithmetic is what a wavefront waits for (with 16 and with 4 a workgroup: 24 x 8388608 elements in fp32 1011 and 1020 us, in 8 bits
// 562 and 561; ResNet-50's tensors in fp32 135 and 132, in 8 bits 105 and 91).
constexpr int adam_tile(int bits) { return bits == 8 ? 4 : 16; }
constexpr int64_t kAdamLaunch = (int64_t)1 << 22;     // tiles of a launch: its threads are counted in 32 bits
constexpr int64_t kAdamPart = (int64_t)1 << 31;       // elements of a tensor in one launch: counted in 32 bits, whole tiles

// The tensors of a launch, by value: as many as leave its arguments below 4 KB.
template <int BITS>
struct AdamTensors;

template <>
struct AdamTensors<32> {
    static constexpr int kMost = 82;
    void* p[kMost];
    const void* g[kMost];
    void *m[kMost], *v[kMost];
    uint16_t* copy[kMost];         // bf16 copy of an fp32 parameter, or null
    uint32_t n[kMost];
    uint32_t first[kMost];         // first tile of a tensor, counted in the launch
};

template <>
struct AdamTensors<8> {
    static constexpr int kMost = 58;
    void* p[kMost];
    const void* g[kMost];
    void *m[kMost], *v[kMost];
    uint16_t* copy[kMost];
    uint32_t n[kMost];
    uint32_t first[kMost];
    float *m_scale[kMost], *v_scale[kMost];
    uint32_t block[kMost];         // its first block, counted in the call
};

template <int BITS>
struct AdamArgs {
    AdamTensors<BITS> t;
    int count;
    uint32_t mix;
    const float* grad_scale;
    // what the formula takes, computed in 64 bits
    float b1, one_b1, b2, one_b2, decay, rate, inv_root_bc2, eps;
};
static_assert(sizeof(AdamArgs<32>) <= 4096 && sizeof(AdamArgs<8>) <= 4096, "a launch's arguments");

template <int BITS>
int adamw_launch(const AdamArgs<BITS>& a, uint32_t tiles, int param_dt, int grad_dt, hipStream_t stream);

}  // namespace sdgp
