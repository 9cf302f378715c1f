// extern "C" boundary of the operators on packed sequences: attention between a model's linear layers, the positions of its
// queries and keys, and the losses behind its token log probabilities.  Argument validation and dispatch; every check happens
// before the first launch.
#include <math.h>

#include "attention_api.h"

namespace {

constexpr int64_t kMostRows = (int64_t)1 << 30;      // tokens times heads: counted in 32 bits
constexpr int64_t kMostStride = (int64_t)1 << 40;
constexpr int kMostHead = 128;

bool valid_dtype(int dt) { return dt == SDGP_F32 || dt == SDGP_BF16; }
bool aligned(const void* p, int64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }
int64_t element(int dt) { return dt == SDGP_BF16 ? 2 : 4; }

int check_attention_sizes(int64_t S, int64_t Tq, int64_t Tk, int64_t H, int64_t Hk, int D, int dt) {
    if (!valid_dtype(dt)) return SDGP_ERR_DTYPE;
    if (S < 0 || Tq < 0 || Tk < 0 || H < 1 || Hk < 1 || H % Hk != 0 || D < 1 || D > kMostHead) return SDGP_ERR_SHAPE;
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

size_t sdgp_attention_bwd_workspace(int64_t Tq, int64_t H) {
    if (H < 1 || Tq < 0 || Tq > kMostRows / H) return (size_t)-1;
    return (size_t)(Tq * H) * sizeof(float);
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
    const size_t need = sdgp_attention_bwd_workspace(Tq, H);
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return SDGP_ERR_WORKSPACE;
    return sdgp::attention_bwd_launch_all(c, dO, o, lse, dq, dk, dv, workspace, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
