// Arguments of the losses over sequences of token log probabilities.
#pragma once

#include "common.h"

namespace sdgp {

struct Sequences {
    const float *logp, *ref;
    const uint8_t* mask;           // null: every token of a sequence counts
    const int32_t* offsets;        // null: S sequences of L tokens
    int64_t T;
    int S, L;
};

struct PolicyLoss {
    Sequences s;
    const float *old, *advantages;
    bool each;                     // an advantage a token, not a sequence
    bool by_sequence;              // mean over the sequences' means, not over the tokens
    float kl, low, high;           // low and high bound the ratio
    double log_low, log_high;
};

struct PreferenceLoss {
    Sequences s;
    double beta, margin, smoothing;
    bool average;
};

size_t sequence_loss_workspace(int64_t T, int64_t S);
int policy_loss_launch(const PolicyLoss& p, float* out, float* weights, void* workspace, hipStream_t stream);
int policy_loss_bwd_launch(const PolicyLoss& p, const float* g, const float* weights, float* dlogp, hipStream_t stream);
int preference_loss_launch(const PreferenceLoss& p, float* loss, float* margins, float* weights, void* workspace, hipStream_t stream);
int preference_loss_bwd_launch(const Sequences& s, const float* g, const float* weights, float* dlogp, hipStream_t stream);

}  // namespace sdgp
