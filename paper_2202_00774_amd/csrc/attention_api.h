// What the C boundary hands to the attention kernels' dispatch.
#pragma once

#include "common.h"

namespace sdgp {

struct AttentionCall {
    const void *q, *k, *v;
    const int64_t* strides;   // of a token and of a head: q, k, v
    const int32_t *offsets_q, *offsets_k, *lengths_k;
    int64_t S, Tq, Tk, H, Hk;
    int D, dt, causal;
    float scale;
};

size_t attention_workspace(int64_t S, int64_t Tq, int64_t Tk, int64_t H, int64_t Hk, int D);
size_t attention_bwd_workspace(int64_t S, int64_t Tq, int64_t Tk, int64_t H, int64_t Hk, int D, int dt);
int attention_launch(const AttentionCall& c, void* o, float* lse, void* workspace, hipStream_t stream);
int attention_bwd_launch_all(const AttentionCall& c, const void* d_o, const void* o, const float* lse, void* dq, void* dk, void* dv,
                             void* workspace, hipStream_t stream);

}  // namespace sdgp
