// extern "C" boundary of the operators around the pruned layers: the loss of a language model's last layer, the norms
// between layers, the optimizer step.  Argument validation and dispatch; every check happens before the first launch.
#include <cmath>

#include "adamw.h"

namespace sdgp {
size_t token_logprobs_workspace(int64_t rows, int64_t V, int dt, int top);
int token_logprobs_launch(const void* logits, int64_t ld, const void* tokens, int token_bits, float* logp, float* entropy,
                          float* top_logp, int64_t* top_ids, float* stats, int64_t rows, int64_t V, int dt, int top, float scale,
                          void* workspace, hipStream_t stream);
int token_logprobs_bwd_launch(const void* logits, int64_t ld, const void* tokens, int token_bits, const float* stats,
                              const float* entropy, const float* g_logp, const float* g_entropy, void* dlogits, int64_t ld_out,
                              int64_t rows, int64_t V, int dt, float scale, hipStream_t stream);
int block_norm_bwd_no_rows(void* dgate, int64_t gate_elements, int dt, float* dw_post, float* dw_pre, int64_t D, hipStream_t stream);
size_t block_norm_bwd_workspace(int64_t rows, int64_t D, int64_t groups, int dt);
int block_norm_launch(const void* x, const void* u, const void* gate, const void* w_post, const void* w_pre, void* y, void* h,
                      float* stats, int64_t rows, int64_t D, int64_t groups, int dt, int wdt, float residual_scale, float eps,
                      hipStream_t stream);
int block_norm_bwd_launch(const void* dy, const void* dh, const void* y, const void* u, const void* gate, const void* w_post,
                          const void* w_pre, const float* stats, void* dx, void* du, void* dgate, float* dw_post, float* dw_pre,
                          int64_t rows, int64_t D, int64_t groups, int dt, int wdt, float residual_scale, void* workspace,
                          hipStream_t stream);
}  // namespace sdgp

namespace {

constexpr int64_t kMaxElements = (int64_t)1 << 40;
constexpr int kMaxTop = 64;                      // a wavefront's lanes
constexpr int64_t kMaxWidth = (int64_t)1 << 30;  // logits of a row: counted in 32 bits
constexpr int64_t kMaxChannels = (int64_t)1 << 20;

bool valid_dtype(int dt) { return dt == SDGP_F32 || dt == SDGP_BF16; }
int64_t element(int dt) { return dt == SDGP_BF16 ? 2 : 4; }
bool aligned(const void* p, int64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

// rows x width within the counted range; a row stride of at least the width.
int check_rows(int64_t rows, int64_t width, int64_t ld, int dt) {
    if (!valid_dtype(dt)) return SDGP_ERR_DTYPE;
    if (rows < 0 || width < 1 || width > kMaxWidth || ld < width) return SDGP_ERR_SHAPE;
    if (rows > kMaxElements / ld) return SDGP_ERR_SHAPE;
    return SDGP_OK;
}

int check_logits(int64_t rows, int64_t V, int64_t ld, int dt, int top) {
    const int rc = check_rows(rows, V, ld, dt);
    if (rc != SDGP_OK) return rc;
    return top < 0 || top > kMaxTop || top > V ? SDGP_ERR_SHAPE : SDGP_OK;
}

bool scale_fits(float x) { return x > 0.0f && x <= 0x1p127f; }   // times log2(e) it has an fp32 value

// groups gates for rows rows: none, or a number that divides the rows.
int check_norm(int64_t rows, int64_t D, int64_t groups, int dt, int wdt) {
    const int rc = check_rows(rows, D, D, dt);
    if (rc != SDGP_OK) return rc;
    if (!valid_dtype(wdt)) return SDGP_ERR_DTYPE;
    if (D > kMaxChannels) return SDGP_ERR_SHAPE;
    return groups < 0 || (groups > 0 && rows % groups != 0) ? SDGP_ERR_SHAPE : SDGP_OK;
}

struct AdamCall {
    int count;
    void* const* params;
    const void* const* grads;
    void* const* exp_avg;
    void* const* exp_avg_sq;
    float* const* exp_avg_scale;
    float* const* exp_avg_sq_scale;
    void* const* copies;
    const int64_t* numel;
    int param_dt, grad_dt;
    hipStream_t stream;
};

// As many launches as the tensors fill.  A tensor longer than a launch counts goes in parts of whole tiles.
template <int BITS>
int adamw_launches(const AdamCall& c, sdgp::AdamArgs<BITS>& a) {
    constexpr int64_t kTile = (int64_t)sdgp::adam_tile(BITS) * sdgp::kAdamBlock;
    int64_t tiles = 0, block = 0;   // tiles of this launch; a tensor's first block, counted in the call
    int k = 0;
    const auto launch = [&] {
        a.count = k;
        const int rc = sdgp::adamw_launch<BITS>(a, (uint32_t)tiles, c.param_dt, c.grad_dt, c.stream);
        tiles = 0, k = 0;
        return rc;
    };
    for (int i = 0; i < c.count; ++i) {
        for (int64_t from = 0; from < c.numel[i];) {
            if (k == sdgp::AdamTensors<BITS>::kMost || tiles == sdgp::kAdamLaunch) {
                const int rc = launch();
                if (rc != SDGP_OK) return rc;
            }
            int64_t part = (sdgp::kAdamLaunch - tiles) * kTile;
            part = part < sdgp::kAdamPart ? part : sdgp::kAdamPart;
            part = part < c.numel[i] - from ? part : c.numel[i] - from;
            auto& t = a.t;
            t.p[k] = static_cast<char*>(c.params[i]) + from * element(c.param_dt);
            t.g[k] = static_cast<const char*>(c.grads[i]) + from * element(c.grad_dt);
            t.m[k] = static_cast<char*>(c.exp_avg[i]) + from * (BITS / 8);
            t.v[k] = static_cast<char*>(c.exp_avg_sq[i]) + from * (BITS / 8);
            t.copy[k] = c.copies ? static_cast<uint16_t*>(c.copies[i]) + from : nullptr;
            t.n[k] = (uint32_t)part;
            t.first[k] = (uint32_t)tiles;
            if constexpr (BITS == 8) {
                const int64_t at = from / sdgp::kAdamBlock;
                t.m_scale[k] = c.exp_avg_scale[i] + at;
                t.v_scale[k] = c.exp_avg_sq_scale[i] + at;
                t.block[k] = (uint32_t)(block + at);
            }
            tiles += (part + kTile - 1) / kTile;
            ++k;
            from += part;
        }
        block += (c.numel[i] + sdgp::kAdamBlock - 1) / sdgp::kAdamBlock;
    }
    return k == 0 ? SDGP_OK : launch();
}

}  // namespace

extern "C" {

size_t sdgp_token_logprobs_workspace(int64_t rows, int64_t V, int dt, int top) {
    if (check_logits(rows, V, V, dt, top) != SDGP_OK) return (size_t)-1;
    return sdgp::token_logprobs_workspace(rows, V, dt, top);
}

int sdgp_token_logprobs(const void* logits, int64_t ld, const void* tokens, int token_bits, float* logp, float* entropy,
                        float* top_logp, int64_t* top_ids, float* stats, int64_t rows, int64_t V, int dt, int top, float scale,
                        void* workspace, size_t workspace_bytes, void* hip_stream) {
    const int rc = check_logits(rows, V, ld, dt, top);
    if (rc != SDGP_OK) return rc;
    if (token_bits != 32 && token_bits != 64) return SDGP_ERR_DTYPE;
    if (!scale_fits(scale)) return SDGP_ERR_VALUE;
    if (rows == 0) return SDGP_OK;
    if (!logits || !entropy || !stats || (logp && !tokens) || (top > 0 && (!top_logp || !top_ids))) return SDGP_ERR_NULL;
    if (!aligned(logits, element(dt)) || (logp && !aligned(tokens, token_bits / 8))) return SDGP_ERR_SHAPE;
    const size_t need = sdgp::token_logprobs_workspace(rows, V, dt, top);
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return SDGP_ERR_WORKSPACE;
    return sdgp::token_logprobs_launch(logits, ld, tokens, token_bits, logp, entropy, top_logp, top_ids, stats, rows, V, dt, top, scale,
                                       workspace, static_cast<hipStream_t>(hip_stream));
}

int sdgp_token_logprobs_bwd(const void* logits, int64_t ld, const void* tokens, int token_bits, const float* stats,
                            const float* entropy, const float* g_logp, const float* g_entropy, void* dlogits, int64_t ld_out,
                            int64_t rows, int64_t V, int dt, float scale, void* hip_stream) {
    int rc = check_logits(rows, V, ld, dt, 0);
    if (rc == SDGP_OK) rc = check_logits(rows, V, ld_out, dt, 0);
    if (rc != SDGP_OK) return rc;
    if (token_bits != 32 && token_bits != 64) return SDGP_ERR_DTYPE;
    if (!scale_fits(scale)) return SDGP_ERR_VALUE;
    if (rows == 0) return SDGP_OK;
    if (!logits || !stats || !dlogits || (g_logp && !tokens) || (g_entropy && !entropy) || (!g_logp && !g_entropy)) return SDGP_ERR_NULL;
    if (!aligned(logits, element(dt)) || !aligned(dlogits, element(dt))) return SDGP_ERR_SHAPE;
    if (g_logp && !aligned(tokens, token_bits / 8)) return SDGP_ERR_SHAPE;   // else they are not read
    return sdgp::token_logprobs_bwd_launch(logits, ld, tokens, token_bits, stats, entropy, g_logp, g_entropy, dlogits, ld_out, rows, V,
                                           dt, scale, static_cast<hipStream_t>(hip_stream));
}

int sdgp_block_norm(const void* x, const void* u, const void* gate, const void* w_post, const void* w_pre, void* y, void* h,
                    float* stats, int64_t rows, int64_t D, int64_t groups, int dt, int wdt, float residual_scale, float eps,
                    void* hip_stream) {
    const int rc = check_norm(rows, D, groups, dt, wdt);
    if (rc != SDGP_OK) return rc;
    if (!std::isfinite(residual_scale) || !std::isfinite(eps) || eps < 0.0f) return SDGP_ERR_VALUE;
    if (rows == 0) return SDGP_OK;
    if (!u && (gate || w_post || y)) return SDGP_ERR_NULL;      // nothing behind a block without its output
    if ((groups > 0) != (gate != nullptr)) return SDGP_ERR_NULL;
    if (!x || !stats || (u && !y) || (!u && !h) || (w_pre && !h)) return SDGP_ERR_NULL;
    for (const void* p : {x, u, gate, (const void*)y, (const void*)h})
        if (!aligned(p, element(dt))) return SDGP_ERR_SHAPE;
    for (const void* p : {w_post, w_pre})
        if (!aligned(p, element(wdt))) return SDGP_ERR_SHAPE;
    return sdgp::block_norm_launch(x, u, gate, w_post, w_pre, y, h, stats, rows, D, groups, dt, wdt, residual_scale, eps,
                                   static_cast<hipStream_t>(hip_stream));
}

size_t sdgp_block_norm_bwd_workspace(int64_t rows, int64_t D, int64_t groups, int dt) {
    if (check_norm(rows, D, groups, dt, SDGP_F32) != SDGP_OK) return (size_t)-1;
    return rows == 0 ? 0 : sdgp::block_norm_bwd_workspace(rows, D, groups, dt);
}

int sdgp_block_norm_bwd(const void* dy, const void* dh, const void* y, const void* u, const void* gate, const void* w_post,
                        const void* w_pre, const float* stats, void* dx, void* du, void* dgate, float* dw_post, float* dw_pre,
                        int64_t rows, int64_t D, int64_t groups, int dt, int wdt, float residual_scale, void* workspace,
                        size_t workspace_bytes, void* hip_stream) {
    const int rc = check_norm(rows, D, groups, dt, wdt);
    if (rc != SDGP_OK) return rc;
    if (!std::isfinite(residual_scale)) return SDGP_ERR_VALUE;
    if (rows == 0) {   // the sums over no rows; tensors without elements may have no address
        return sdgp::block_norm_bwd_no_rows(dgate, groups * D, dt, dw_post, dw_pre, D, static_cast<hipStream_t>(hip_stream));
    }
    if (!u && (gate || w_post || du || dgate || dw_post)) return SDGP_ERR_NULL;
    if ((groups > 0) != (gate != nullptr)) return SDGP_ERR_NULL;
    // a weight's gradient is the weight's: none without it
    if ((w_post != nullptr) != (dw_post != nullptr) || (w_pre != nullptr) != (dw_pre != nullptr) || (gate != nullptr) != (dgate != nullptr))
        return SDGP_ERR_NULL;
    if (!dh && (w_pre || !dy)) return SDGP_ERR_NULL;
    if (!y || !stats || !dx || (u && !du)) return SDGP_ERR_NULL;
    for (const void* p : {dy, dh, y, u, gate, (const void*)dx, (const void*)du, (const void*)dgate})
        if (!aligned(p, element(dt))) return SDGP_ERR_SHAPE;
    for (const void* p : {w_post, w_pre})
        if (!aligned(p, element(wdt))) return SDGP_ERR_SHAPE;
    const size_t need = sdgp::block_norm_bwd_workspace(rows, D, groups, dt);
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return SDGP_ERR_WORKSPACE;
    return sdgp::block_norm_bwd_launch(dy, dh, y, u, gate, w_post, w_pre, stats, dx, du, dgate, dw_post, dw_pre, rows, D, groups, dt, wdt,
                                       residual_scale, workspace, static_cast<hipStream_t>(hip_stream));
}

int sdgp_adamw_step(int count, void* const* params, const void* const* grads, void* const* exp_avg, void* const* exp_avg_sq,
                    float* const* exp_avg_scale, float* const* exp_avg_sq_scale, void* const* copies, const int64_t* numel,
                    int param_dt, int grad_dt, int state_bits, double lr, double beta1, double beta2, double eps,
                    double weight_decay, int64_t step, const float* grad_scale, uint64_t seed, void* hip_stream) {
    if (!valid_dtype(param_dt) || !valid_dtype(grad_dt) || (state_bits != 32 && state_bits != 8)) return SDGP_ERR_DTYPE;
    if (count < 0) return SDGP_ERR_SHAPE;
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !std::isfinite(lr) || lr < 0.0 || !std::isfinite(eps) ||
        eps < 0.0 || !std::isfinite(weight_decay) || weight_decay < 0.0 || step < 1)
        return SDGP_ERR_VALUE;
    if (count == 0) return SDGP_OK;
    if (!params || !grads || !exp_avg || !exp_avg_sq || !numel || (state_bits == 8 && (!exp_avg_scale || !exp_avg_sq_scale)))
        return SDGP_ERR_NULL;
    if (copies && param_dt != SDGP_F32) return SDGP_ERR_DTYPE;
    int64_t blocks = 0;
    for (int i = 0; i < count; ++i) {
        if (numel[i] < 0 || numel[i] > kMaxElements) return SDGP_ERR_SHAPE;
        blocks += (numel[i] + sdgp::kAdamBlock - 1) / sdgp::kAdamBlock;
        if (blocks > kMaxElements / sdgp::kAdamBlock) return SDGP_ERR_SHAPE;
        if (numel[i] == 0) continue;
        if (!params[i] || !grads[i] || !exp_avg[i] || !exp_avg_sq[i] || (copies && !copies[i])) return SDGP_ERR_NULL;
        if (state_bits == 8 && (!exp_avg_scale[i] || !exp_avg_sq_scale[i])) return SDGP_ERR_NULL;
        if (!aligned(params[i], element(param_dt)) || !aligned(grads[i], element(grad_dt)) || (copies && !aligned(copies[i], 2)))
            return SDGP_ERR_SHAPE;
        if (state_bits == 32 && (!aligned(exp_avg[i], 4) || !aligned(exp_avg_sq[i], 4))) return SDGP_ERR_SHAPE;
        if (state_bits == 8 && (!aligned(exp_avg_scale[i], 4) || !aligned(exp_avg_sq_scale[i], 4))) return SDGP_ERR_SHAPE;
    }
    if (blocks == 0) return SDGP_OK;
    // The step's number and seed go to the kernel by value: a graph would make this one step again in every replay.  (The default
    // stream is never captured, and asking takes 1 us of the smallest steps' 11.)
    hipStreamCaptureStatus capturing = hipStreamCaptureStatusNone;
    if (hip_stream != nullptr && hipStreamIsCapturing(static_cast<hipStream_t>(hip_stream), &capturing) != hipSuccess) {
        (void)hipGetLastError();
        return SDGP_ERR_HIP;
    }
    if (capturing != hipStreamCaptureStatusNone) return SDGP_ERR_VALUE;
    const AdamCall c = {count, params, grads, exp_avg, exp_avg_sq, exp_avg_scale, exp_avg_sq_scale, copies, numel, param_dt, grad_dt,
                        static_cast<hipStream_t>(hip_stream)};
    const double bc1 = 1.0 - std::pow(beta1, (double)step), bc2 = 1.0 - std::pow(beta2, (double)step);
    const auto rates = [&](auto& a) {
        a.mix = sdgp::seed_mix(seed);
        a.grad_scale = grad_scale;
        a.b1 = (float)beta1, a.one_b1 = (float)(1.0 - beta1), a.b2 = (float)beta2, a.one_b2 = (float)(1.0 - beta2);
        a.decay = (float)(1.0 - lr * weight_decay);
        a.rate = (float)(lr / bc1);
        a.inv_root_bc2 = (float)(1.0 / std::sqrt(bc2));
        a.eps = (float)eps;
    };
    if (state_bits == 8) {
        sdgp::AdamArgs<8> a;
        rates(a);
        return adamw_launches(c, a);
    }
    sdgp::AdamArgs<32> a;
    rates(a);
    return adamw_launches(c, a);
}

}  // extern "C"
