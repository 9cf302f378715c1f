// extern "C" boundary of the operators on packed sequences: attention between a model's linear layers, the positions of its
// queries and keys, and the losses behind its token log probabilities.  Argument validation and dispatch; every check happens
// before the first launch.
#include <math.h>

#include "attention_api.h"
#include "rotary.h"
#include "sequence_loss.h"

namespace {

constexpr int64_t kMostRows = (int64_t)1 << 30;      // tokens times heads: counted in 32 bits
constexpr int64_t kMostStride = (int64_t)1 << 40;
constexpr int kMostHead = 128;
constexpr int64_t kMostHeads = 65536;
constexpr int64_t kMostGrid = 0xFFFFFF;              // workgroups of 256 threads: a launch counts threads in 32 bits

bool valid_dtype(int dt) { return dt == SDGP_F32 || dt == SDGP_BF16; }
bool aligned(const void* p, int64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }
int64_t element(int dt) { return dt == SDGP_BF16 ? 2 : 4; }

int check_attention_sizes(int64_t S, int64_t Tq, int64_t Tk, int64_t H, int64_t Hk, int D, int dt) {
    if (!valid_dtype(dt)) return SDGP_ERR_DTYPE;
    if (S < 0 || Tq < 0 || Tk < 0 || H < 1 || H > kMostHeads || Hk < 1 || H % Hk != 0 || D < 1 || D > kMostHead) return SDGP_ERR_SHAPE;
    if (S > kMostRows / H || Tq > kMostRows / H || Tk > kMostRows / H) return SDGP_ERR_SHAPE;
    return SDGP_OK;
}

int check_attention(const sdgp::AttentionCall& c) {
    const int rc = check_attention_sizes(c.S, c.Tq, c.Tk, c.H, c.Hk, c.D, c.dt);
    if (rc != SDGP_OK) return rc;
    if (!(c.scale >= 1e-30f && c.scale <= 1e30f)) return SDGP_ERR_VALUE;
    if ((c.offsets_q != nullptr) != (c.offsets_k != nullptr)) return SDGP_ERR_NULL;
    if (c.offsets_q != nullptr && c.lengths_k != nullptr) return SDGP_ERR_VALUE;       // packed keys have their lengths
    if (c.offsets_q == nullptr && (c.S == 0 ? c.Tq + c.Tk > 0 : c.Tq % c.S != 0 || c.Tk % c.S != 0)) return SDGP_ERR_SHAPE;
    if (c.strides == nullptr) return SDGP_ERR_NULL;
    for (int i = 0; i < 6; ++i)
        if (c.strides[i] < 0 || c.strides[i] > kMostStride) return SDGP_ERR_SHAPE;
    for (const void* p : {(const void*)c.offsets_q, (const void*)c.offsets_k, (const void*)c.lengths_k})
        if (!aligned(p, 4)) return SDGP_ERR_SHAPE;
    if ((c.Tq > 0 && !c.q) || (c.Tk > 0 && (!c.k || !c.v))) return SDGP_ERR_NULL;
    for (const void* p : {c.q, c.k, c.v})
        if (!aligned(p, element(c.dt))) return SDGP_ERR_SHAPE;
    return SDGP_OK;
}

constexpr int64_t kMostTokens = kMostGrid * 1024, kMostSequences = kMostGrid * 4;   // a workgroup's

// The sequences' tokens, without their addresses.
int check_sequences(int64_t T, int64_t S, bool packed) {
    if (T < 0 || S < 0 || S > kMostSequences || T > kMostTokens) return SDGP_ERR_SHAPE;
    if (packed ? T > 0x7FFFFFFF : S == 0 ? T > 0 : T % S != 0 || T / S > 0x7FFFFFFF) return SDGP_ERR_SHAPE;   // offsets have 32 bits
    return SDGP_OK;
}

int check_tokens(const sdgp::Sequences& s) {
    if (s.T > 0 && !s.logp) return SDGP_ERR_NULL;
    return aligned(s.logp, 4) && aligned(s.ref, 4) && aligned(s.offsets, 4) ? SDGP_OK : SDGP_ERR_SHAPE;
}

sdgp::Sequences sequences_of(const float* logp, const float* ref, const uint8_t* mask, const int32_t* offsets, int64_t T, int64_t S) {
    return {logp, ref, mask, offsets, T, (int)S, S > 0 ? (int)(T / S < 0x7FFFFFFF ? T / S : 0x7FFFFFFF) : 0};
}

int check_policy(const sdgp::Sequences& s, int64_t S, const float* old, const float* advantages, int each, double low, double high, float kl) {
    int rc = check_sequences(s.T, S, s.offsets != nullptr);
    if (rc != SDGP_OK) return rc;
    if (!(low >= 0.0 && low <= 1.0) || !(high >= 0.0) || !isfinite(kl) || kl < 0.0f || (kl > 0.0f && s.T > 0 && !s.ref)) return SDGP_ERR_VALUE;
    rc = check_tokens(s);
    if (rc != SDGP_OK) return rc;
    if ((s.T > 0 && !old) || ((each ? s.T : S) > 0 && !advantages)) return SDGP_ERR_NULL;
    return aligned(old, 4) && aligned(advantages, 4) ? SDGP_OK : SDGP_ERR_SHAPE;
}

sdgp::PolicyLoss policy_of(const sdgp::Sequences& s, const float* old, const float* advantages, int each, int by_sequence, double low, double high, float kl) {
    return {s, old, advantages, each != 0, by_sequence != 0, kl, (float)(1.0 - low), (float)(1.0 + high), log1p(-low), log1p(high)};
}

}  // namespace

extern "C" {

size_t sdgp_attention_workspace(int64_t sequences, int64_t Tq, int64_t Tk, int64_t H, int64_t Hk, int D, int dt) {
    if (check_attention_sizes(sequences, Tq, Tk, H, Hk, D, dt) != SDGP_OK) return (size_t)-1;
    return sdgp::attention_workspace(sequences, Tq, Tk, H, Hk, D);
}

int sdgp_attention(const void* q, const void* k, const void* v, const int64_t* strides, const int32_t* offsets_q,
                   const int32_t* offsets_k, const int32_t* lengths_k, int64_t sequences, void* o, float* lse, int64_t Tq, int64_t Tk,
                   int64_t H, int64_t Hk, int D, int dt, int causal, float scale, void* workspace, size_t workspace_bytes,
                   void* hip_stream) {
    const sdgp::AttentionCall c = {q, k, v, strides, offsets_q, offsets_k, lengths_k, sequences, Tq, Tk, H, Hk, D, dt, causal != 0, scale};
    const int rc = check_attention(c);
    if (rc != SDGP_OK) return rc;
    if (Tq == 0) return SDGP_OK;
    if (!o || !lse) return SDGP_ERR_NULL;
    if (!aligned(o, element(dt)) || !aligned(lse, 4)) return SDGP_ERR_SHAPE;
    const size_t need = sdgp::attention_workspace(sequences, Tq, Tk, H, Hk, D);
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return SDGP_ERR_WORKSPACE;
    return sdgp::attention_launch(c, o, lse, workspace, static_cast<hipStream_t>(hip_stream));
}

size_t sdgp_attention_bwd_workspace(int64_t sequences, int64_t Tq, int64_t Tk, int64_t H, int64_t Hk, int D, int dt) {
    if (check_attention_sizes(sequences, Tq, Tk, H, Hk, D, dt) != SDGP_OK) return (size_t)-1;
    return sdgp::attention_bwd_workspace(sequences, Tq, Tk, H, Hk, D, dt);
}

int sdgp_attention_bwd(const void* dO, const void* q, const void* k, const void* v, const void* o, const float* lse,
                       const int64_t* strides, const int32_t* offsets_q, const int32_t* offsets_k, int64_t sequences, void* dq, void* dk,
                       void* dv, int64_t Tq, int64_t Tk, int64_t H, int64_t Hk, int D, int dt, int causal, float scale, void* workspace,
                       size_t workspace_bytes, void* hip_stream) {
    const sdgp::AttentionCall c = {q, k, v, strides, offsets_q, offsets_k, nullptr, sequences, Tq, Tk, H, Hk, D, dt, causal != 0, scale};
    const int rc = check_attention(c);
    if (rc != SDGP_OK) return rc;
    if ((Tq > 0 && (!dO || !o || !lse || !dq)) || (Tk > 0 && (!dk || !dv))) return SDGP_ERR_NULL;
    for (const void* p : {dO, o, (const void*)dq, (const void*)dk, (const void*)dv})
        if (!aligned(p, element(dt))) return SDGP_ERR_SHAPE;
    if (!aligned(lse, 4)) return SDGP_ERR_SHAPE;
    const size_t need = sdgp::attention_bwd_workspace(sequences, Tq, Tk, H, Hk, D, dt);
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return SDGP_ERR_WORKSPACE;
    return sdgp::attention_bwd_launch_all(c, dO, o, lse, dq, dk, dv, workspace, static_cast<hipStream_t>(hip_stream));
}

int sdgp_rotary(const void* q, const void* k, void* q_out, void* k_out, const int64_t* strides, const void* positions, int position_bits,
                const float* freqs, const int32_t* axis_pairs, int axes, int64_t T, int64_t H, int64_t Hk, int64_t D, int dt,
                int interleaved, int inverse, void* hip_stream) {
    if (!valid_dtype(dt) || (position_bits != 32 && position_bits != 64)) return SDGP_ERR_DTYPE;
    if (T < 0 || H < 1 || Hk < 0 || D < 2 || D > 4096 || H > 4096 || Hk > 4096 || axes < 1 || axes > sdgp::kMaxAxes) return SDGP_ERR_SHAPE;
    if (T > 0x7FFFFFFF || (H + Hk) * D > (int64_t)1 << 22) return SDGP_ERR_SHAPE;
    if (!strides || !axis_pairs) return SDGP_ERR_NULL;
    sdgp::Rotary a = {};
    int64_t pairs = 0;
    for (int i = 0; i < axes; ++i) {
        if (axis_pairs[i] < 1) return SDGP_ERR_SHAPE;
        pairs += axis_pairs[i];
        if (2 * pairs > D) return SDGP_ERR_SHAPE;
        a.end[i] = (int)pairs;
    }
    for (int i = 0; i < 8; ++i)
        if (strides[i] < 0 || strides[i] > kMostStride) return SDGP_ERR_SHAPE;
    if (T == 0) return SDGP_OK;
    if (!q || !q_out || !positions || !freqs || (Hk > 0) != (k != nullptr) || (Hk > 0) != (k_out != nullptr)) return SDGP_ERR_NULL;
    for (const void* p : {q, k, (const void*)q_out, (const void*)k_out})
        if (!aligned(p, element(dt))) return SDGP_ERR_SHAPE;
    if (!aligned(positions, position_bits / 8) || !aligned(freqs, 4)) return SDGP_ERR_SHAPE;
    // every output element is written once
    if ((T > 1 && strides[4] < D) || (H > 1 && strides[5] < D) || (Hk > 0 && T > 1 && strides[6] < D) || (Hk > 1 && strides[7] < D)) return SDGP_ERR_SHAPE;
    if ((T + sdgp::rotary_tokens(pairs) - 1) / sdgp::rotary_tokens(pairs) > kMostGrid) return SDGP_ERR_SHAPE;
    a.q = q, a.k = k, a.q_out = q_out, a.k_out = k_out;
    a.q_token = strides[0], a.q_head = strides[1], a.k_token = strides[2], a.k_head = strides[3];
    a.q_out_token = strides[4], a.q_out_head = strides[5], a.k_out_token = strides[6], a.k_out_head = strides[7];
    a.positions = positions, a.freqs = freqs, a.T = T, a.H = (int)H, a.Hk = (int)Hk, a.D = (int)D, a.F = (int)pairs, a.axes = axes;
    a.position_bits = position_bits, a.inverse = inverse != 0;
    return sdgp::rotary_launch(a, dt, interleaved != 0, static_cast<hipStream_t>(hip_stream));
}

size_t sdgp_sequence_loss_workspace(int64_t T, int64_t sequences) {
    if (T < 0 || sequences < 0 || sequences > kMostSequences || T > kMostTokens) return (size_t)-1;
    return sdgp::sequence_loss_workspace(T, sequences);
}

int sdgp_policy_loss(const float* logp, const float* old_logp, const float* ref_logp, const float* advantages, int each,
                     const uint8_t* mask, const int32_t* offsets, int64_t sequences, int64_t T, double low, double high, float kl,
                     int by_sequence, float* out, float* weights, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const sdgp::Sequences s = sequences_of(logp, ref_logp, mask, offsets, T, sequences);
    const int rc = check_policy(s, sequences, old_logp, advantages, each, low, high, kl);
    if (rc != SDGP_OK) return rc;
    if (!out || (sequences > 0 && !weights)) return SDGP_ERR_NULL;
    if (!aligned(out, 4) || !aligned(weights, 4)) return SDGP_ERR_SHAPE;
    const size_t need = sdgp::sequence_loss_workspace(T, sequences);
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return SDGP_ERR_WORKSPACE;
    return sdgp::policy_loss_launch(policy_of(s, old_logp, advantages, each, by_sequence, low, high, kl), out, weights, workspace,
                                    static_cast<hipStream_t>(hip_stream));
}

int sdgp_policy_loss_bwd(const float* g, const float* weights, const float* logp, const float* old_logp, const float* ref_logp,
                         const float* advantages, int each, const uint8_t* mask, const int32_t* offsets, int64_t sequences, int64_t T,
                         double low, double high, float kl, float* dlogp, void* hip_stream) {
    sdgp::Sequences s = sequences_of(logp, ref_logp, mask, offsets, T, sequences);
    const int rc = check_policy(s, sequences, old_logp, advantages, each, low, high, kl);
    if (rc != SDGP_OK) return rc;
    if (T == 0) return SDGP_OK;
    if (!g || (sequences > 0 && !weights) || !dlogp) return SDGP_ERR_NULL;
    if (!aligned(g, 4) || !aligned(weights, 4) || !aligned(dlogp, 4)) return SDGP_ERR_SHAPE;
    s.ref = kl > 0.0f ? s.ref : nullptr;                                // nothing of it is in the gradient
    return sdgp::policy_loss_bwd_launch(policy_of(s, old_logp, advantages, each, 0, low, high, kl), g, weights, dlogp,
                                        static_cast<hipStream_t>(hip_stream));
}

int sdgp_preference_loss(const float* logp, const float* ref_logp, const uint8_t* mask, const int32_t* offsets, int64_t sequences,
                         int64_t T, double beta, double margin, double smoothing, int average, float* loss, float* margins,
                         float* weights, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const sdgp::Sequences s = sequences_of(logp, ref_logp, mask, offsets, T, sequences);
    int rc = check_sequences(T, sequences, offsets != nullptr);
    if (rc != SDGP_OK) return rc;
    if (sequences % 2 != 0) return SDGP_ERR_SHAPE;
    if (!isfinite(beta) || !isfinite(margin) || !(smoothing >= 0.0 && smoothing < 1.0)) return SDGP_ERR_VALUE;
    rc = check_tokens(s);
    if (rc != SDGP_OK) return rc;
    if (!loss || (sequences > 0 && (!margins || !weights))) return SDGP_ERR_NULL;
    if (!aligned(loss, 4) || !aligned(margins, 4) || !aligned(weights, 4)) return SDGP_ERR_SHAPE;
    const size_t need = sdgp::sequence_loss_workspace(T, sequences);
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return SDGP_ERR_WORKSPACE;
    return sdgp::preference_loss_launch({s, beta, margin, smoothing, average != 0}, loss, margins, weights, workspace,
                                        static_cast<hipStream_t>(hip_stream));
}

int sdgp_preference_loss_bwd(const float* g, const float* weights, const uint8_t* mask, const int32_t* offsets, int64_t sequences,
                             int64_t T, float* dlogp, void* hip_stream) {
    const int rc = check_sequences(T, sequences, offsets != nullptr);
    if (rc != SDGP_OK) return rc;
    if (T == 0) return SDGP_OK;
    if (!g || (sequences > 0 && !weights) || !dlogp) return SDGP_ERR_NULL;
    if (!aligned(g, 4) || !aligned(weights, 4) || !aligned(dlogp, 4) || !aligned(offsets, 4)) return SDGP_ERR_SHAPE;
    return sdgp::preference_loss_bwd_launch(sequences_of(nullptr, nullptr, mask, offsets, T, sequences), g, weights, dlogp,
                                            static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
