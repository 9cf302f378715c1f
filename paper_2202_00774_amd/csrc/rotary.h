// Arguments of the rotary kernel.
#pragma once

#include "common.h"
#include "fastdiv.h"

namespace sdgp {

constexpr int kMaxAxes = 8;

struct Rotary {
    const void *q, *k;
    void *q_out, *k_out;
    int64_t q_token, q_head, k_token, k_head, q_out_token, q_out_head, k_out_token, k_out_head;   // strides in elements
    const void* positions;    // [T, axes]
    const float* freqs;       // [F]
    int64_t T;
    int H, Hk, D, F, axes, position_bits;
    int end[kMaxAxes];        // pairs of the axes up to this one
    bool inverse;
    // of the launch: tokens a workgroup, chunks of 16 bytes a head and a token
    int tokens, turned, per_head, per_token;
    FastDiv by_pairs, by_head, by_token;
};

// Tokens of a workgroup: a sine and cosine a thread.
constexpr int rotary_tokens(int64_t pairs) { return pairs > 256 ? 1 : (int)(256 / pairs); }

int rotary_launch(Rotary a, int dt, bool interleaved, hipStream_t stream);

}  // namespace sdgp
