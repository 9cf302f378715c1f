// Losses over sequences of token log probabilities, and their gradients.
//
//   policy      r = exp(logp - old);  l = -min(r A, clip(r, 1 - low, 1 + high) A) + kl (e^x - 1 - x),  x = ref - logp
//               loss = mean of l over the tokens that count, or the mean over sequences of their means
//               dl/dlogp = -r A where the ratio is not cut, else 0;  - kl (e^x - 1)
//   preference  score = beta * sum (or mean) of logp - ref;  z = score(2 i) - score(2 i + 1) - margin
//               loss = mean over pairs of -(1 - smoothing) ln sigma(z) - smoothing ln sigma(-z)
// Whether a ratio is cut is decided on logp - old in 64 bits, which is exact, so it does not hang on the exponential's last bit.
//
// Bound by memory and, for small batches, by launches.  A wavefront takes a chunk of 256 tokens and leaves the sums of each
// sequence's part of it in a slot of its own: chunk + sequence, different for any two parts.  Then a wavefront a sequence adds
// its slots, and one workgroup the sequences.  All in 64 bits and a fixed order: the mean of millions of terms of both signs
// loses nothing.  Small batches do all three steps in one launch.
#include "rows.h"
#include "sequence_loss.h"

namespace sdgp {

namespace {

constexpr int kBlock = 256, kWaves = kBlock / 64, kChunk = 256, kTerms = 4, kFinish = 1024;
constexpr int kOneLaunchSequences = 128;
// Tokens of batches that one workgroup takes through all three steps.  The policy loss's wavefronts should have one chunk each.
template <class Loss>
constexpr int64_t one_launch_tokens();
template <>
constexpr int64_t one_launch_tokens<PolicyLoss>() { return 16 * kChunk; }
template <>
constexpr int64_t one_launch_tokens<PreferenceLoss>() { return 64 * kChunk; }

struct Span {
    int64_t begin, end;
};

__device__ __forceinline__ Span span_of(const Sequences& s, int i) {
    if (s.offsets == nullptr) return {(int64_t)i * s.L, (int64_t)(i + 1) * s.L};
    const int64_t a = s.offsets[i], b = s.offsets[i + 1];
    Span r;
    r.begin = a < 0 ? 0 : a > s.T ? s.T : a;
    r.end = b < r.begin ? r.begin : b > s.T ? s.T : b;
    return r;
}

// The first sequence that ends behind token t (S: none), of one t a wavefront, whose lanes look at 64 of them at once (one by one in
// halves the dependent loads take 22 instead of 19 us for 3.8 million tokens of 512 sequences).
__device__ __forceinline__ int sequence_behind(const Sequences& s, int64_t t) {
    if (s.offsets == nullptr) return s.L == 0 ? s.S : t / s.L < s.S ? (int)(t / s.L) : s.S;
    int lo = 0, hi = s.S;
    while (lo < hi) {
        const int step = (hi - lo + 63) / 64, mine = lo + (int)(threadIdx.x & 63) * step + step - 1, at = mine < hi ? mine : hi - 1;
        const uint64_t past = __ballot(s.offsets[at + 1] > t);
        if (past == 0) return hi;
        lo += __builtin_ctzll(past) * step;
        hi = lo + step - 1 < hi ? lo + step - 1 : hi - 1;
    }
    return lo;
}

template <int CTRL>
__device__ __forceinline__ double lane_swap64(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t low = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, 0xF, 0xF, true);
    const uint32_t high = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, 0xF, 0xF, true);
    return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}

__device__ __forceinline__ double lane_value64(double v, int lane) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t low = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane), high = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}

// In every lane: pairs, fours, a DPP row mirrored in halves and whole, then the four rows (by way of LDS 33 instead of 26 us for
// 64 sequences of up to 200 tokens).
__device__ __forceinline__ double sum_over_wave(double v) {
    v += lane_swap64<0xB1>(v);
    v += lane_swap64<0x4E>(v);
    v += lane_swap64<0x141>(v);
    v += lane_swap64<0x140>(v);
    return (lane_value64(v, 0) + lane_value64(v, 16)) + (lane_value64(v, 32) + lane_value64(v, 48));
}

// What a token's loss and slope (dl/dlogp) take that does not hang on its advantage.
struct TokenTerms {
    double d;                      // logp - old
    float ratio, kl, rise;         // e^d; e^x - 1 - x and e^x - 1
};

__device__ __forceinline__ TokenTerms token_terms(const PolicyLoss& p, float logp, float old, float ref) {
    TokenTerms t;
    t.d = (double)logp - (double)old;
    t.ratio = expf((float)t.d);
    t.kl = t.rise = 0.0f;
    if (p.s.ref != nullptr) {
        // e^x - 1 - x: its series where the differences would cancel (what is left out, from x^11 on, is at most 1.05 x 2^-24 of it, at x = -1)
        const float x = (float)((double)ref - (double)logp);
        float series = 1.0f / 3628800.0f;
        series = __builtin_fmaf(series, x, 1.0f / 362880.0f);
        series = __builtin_fmaf(series, x, 1.0f / 40320.0f);
        series = __builtin_fmaf(series, x, 1.0f / 5040.0f);
        series = __builtin_fmaf(series, x, 1.0f / 720.0f);
        series = __builtin_fmaf(series, x, 1.0f / 120.0f);
        series = __builtin_fmaf(series, x, 1.0f / 24.0f);
        series = __builtin_fmaf(series, x, 1.0f / 6.0f);
        series = __builtin_fmaf(series, x, 0.5f);
        const bool small = fabsf(x) < 1.0f;
        const float e = expf(x) - 1.0f;
        t.kl = small ? series * x * x : e - x;
        t.rise = small ? __builtin_fmaf(series * x, x, x) : e;
    }
    return t;
}

struct PolicyTerms {
    float loss, cut, slope;
};

__device__ __forceinline__ PolicyTerms policy_terms(const PolicyLoss& p, const TokenTerms& t, float A) {
    const bool cut = (A > 0.0f && t.d > p.log_high) || (A < 0.0f && t.d < p.log_low);
    const float ra = A == 0.0f ? 0.0f : t.ratio * A;                   // (an infinite ratio times no advantage)
    PolicyTerms r;
    r.cut = cut ? 1.0f : 0.0f;
    r.loss = (cut ? -A * (A > 0.0f ? p.high : p.low) : -ra) + (p.kl == 0.0f ? 0.0f : p.kl * t.kl);   // (it may be infinite)
    r.slope = (cut ? 0.0f : -ra) - p.kl * t.rise;
    return r;
}

// Four tokens of a lane.
struct Four {
    float logp[4], ref[4], old[4], adv[4];
    bool on[4];
};

__device__ __forceinline__ void load_four(const float* p, int64_t at, int64_t T, float (&v)[4]) {
    const int left = (int)(T - at < 4 ? (T - at < 0 ? 0 : T - at) : 4);
    const auto r = load_row<SDGP_F32>(p + at, 0, left);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = r.get(i);
}

__device__ __forceinline__ void load_mask(const Sequences& s, int64_t at, bool (&on)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) on[i] = at + i < s.T;
    if (s.mask == nullptr) return;
    if (at + 4 <= s.T) {
        typedef uint32_t bytes4 __attribute__((aligned(1), may_alias));
        const uint32_t w = *reinterpret_cast<const bytes4*>(s.mask + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) on[i] = ((w >> (8 * i)) & 0xFFu) != 0;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (on[i]) on[i] = s.mask[at + i] != 0;
    }
}

template <class Loss>
__device__ __forceinline__ Four load_tokens(const Loss& p, int64_t at) {
    Four f;
    const Sequences& s = p.s;
    load_mask(s, at, f.on);
    load_four(s.logp, at, s.T, f.logp);
    if (s.ref != nullptr) load_four(s.ref, at, s.T, f.ref);
    if constexpr (std::is_same<Loss, PolicyLoss>::value) {
        load_four(p.old, at, s.T, f.old);
        if (p.each) load_four(p.advantages, at, s.T, f.adv);
    }
    return f;
}

// A wavefront's chunk: the sums of each sequence's part, to its slot.
template <class Loss>
__device__ __forceinline__ void chunk_sums(const Loss& p, int64_t chunk, double* slots) {
    const Sequences& s = p.s;
    const int lane = threadIdx.x & 63;
    const int64_t begin = chunk * kChunk, end = begin + kChunk < s.T ? begin + kChunk : s.T, at = begin + 4 * lane;
    const Four f = load_tokens(p, at);
    TokenTerms t[4];
    if constexpr (std::is_same<Loss, PolicyLoss>::value)
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = token_terms(p, f.logp[k], f.old[k], f.ref[k]);
    for (int i = sequence_behind(s, begin); i < s.S; ++i) {
        const Span span = span_of(s, i);
        if (span.begin >= end) break;
        double sums[kTerms] = {0.0, 0.0, 0.0, 0.0};
        float A = 0.0f;
        if constexpr (std::is_same<Loss, PolicyLoss>::value) A = p.each ? 0.0f : p.advantages[i];
        int count = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (!(f.on[k] && at + k >= span.begin && at + k < span.end)) continue;
            ++count;
            if constexpr (std::is_same<Loss, PolicyLoss>::value) {
                const PolicyTerms r = policy_terms(p, t[k], p.each ? f.adv[k] : A);
                sums[1] += (double)r.loss, sums[2] += (double)t[k].kl, sums[3] += (double)r.cut;
            } else {
                sums[1] += s.ref != nullptr ? (double)f.logp[k] - (double)f.ref[k] : (double)f.logp[k];
            }
        }
        sums[0] = (double)count;
        constexpr int used = std::is_same<Loss, PolicyLoss>::value ? 4 : 2;
#pragma unroll
        for (int k = 0; k < used; ++k) sums[k] = sum_over_wave(sums[k]);
        if (lane < used) {
            const double v = lane == 0 ? sums[0] : lane == 1 ? sums[1] : lane == 2 ? sums[2] : sums[3];
            slots[(chunk + i) * kTerms + lane] = v;
        }
    }
}

// A wavefront's sequence: its slots' sums (in every lane).
template <int USED>
__device__ __forceinline__ void sequence_sums(const Sequences& s, int i, const double* slots, double (&sums)[kTerms]) {
    const int lane = threadIdx.x & 63;
    const Span span = span_of(s, i);
#pragma unroll
    for (int k = 0; k < kTerms; ++k) sums[k] = 0.0;
    if (span.begin < span.end) {
        const int64_t last = (span.end - 1) / kChunk;
        for (int64_t c = span.begin / kChunk + lane; c <= last; c += 64)
#pragma unroll
            for (int k = 0; k < USED; ++k) sums[k] += slots[(c + i) * kTerms + k];
    }
#pragma unroll
    for (int k = 0; k < USED; ++k) sums[k] = sum_over_wave(sums[k]);
}

// Sums over the workgroup of kFinish threads, the same for every thread.
template <int K>
__device__ __forceinline__ void block_sums(double (&v)[K]) {
    __shared__ double lds[K][kFinish / 64];
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = sum_over_wave(v[k]);
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) lds[k][threadIdx.x / 64] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        v[k] = 0.0;
        for (int w = 0; w < kFinish / 64; ++w) v[k] += lds[k][w];
    }
}

// One workgroup: from the sequences' sums [S, kTerms] to the loss and the sequences' weights in its gradient.
__device__ __forceinline__ void finish(const PolicyLoss& p, const double* sums, float* out, float* weights) {
    double all[5] = {0.0, 0.0, 0.0, 0.0, 0.0};
    double &tokens = all[0], &some = all[1], &loss = all[2], &kl = all[3], &cut = all[4];
    for (int i = threadIdx.x; i < p.s.S; i += kFinish) {
        const double n = sums[i * kTerms];
        if (n == 0.0) continue;
        tokens += n, some += 1.0;
        loss += p.by_sequence ? sums[i * kTerms + 1] / n : sums[i * kTerms + 1];
        kl += sums[i * kTerms + 2], cut += sums[i * kTerms + 3];
    }
    block_sums(all);
    const double share = p.by_sequence ? some : tokens;
    for (int i = threadIdx.x; i < p.s.S; i += kFinish) {
        const double n = sums[i * kTerms];
        weights[i] = n == 0.0 ? 0.0f : (float)(p.by_sequence ? 1.0 / (n * some) : 1.0 / tokens);
    }
    if (threadIdx.x == 0) {
        out[0] = tokens > 0.0 ? (float)(loss / share) : 0.0f;
        out[1] = tokens > 0.0 ? (float)(kl / tokens) : 0.0f;
        out[2] = tokens > 0.0 ? (float)(cut / tokens) : 0.0f;
    }
}

struct PreferenceOut {
    float *loss, *margins, *weights;
};

// sigma(z) without overflow on either side
__device__ __forceinline__ double sigmoid(double z) {
    const double e = exp(-fabs(z));
    return (z >= 0.0 ? 1.0 : e) / (1.0 + e);
}

__device__ __forceinline__ void finish(const PreferenceLoss& p, const double* sums, const PreferenceOut& out) {
    const int pairs = p.s.S / 2;
    double all[1] = {0.0};
    double& loss = all[0];
    for (int i = threadIdx.x; i < pairs; i += kFinish) {
        double each[2], score[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const double n = sums[(2 * i + k) * kTerms];
            each[k] = p.beta / (p.average && n > 1.0 ? n : 1.0);
            score[k] = each[k] * sums[(2 * i + k) * kTerms + 1];
        }
        const double z = score[0] - score[1] - p.margin, tail = log1p(exp(-fabs(z)));
        // -ln sigma(z) = tail + max(-z, 0), -ln sigma(-z) = tail + max(z, 0)
        loss += tail + (z < 0.0 ? (p.smoothing - 1.0) * z : p.smoothing > 0.0 && z > 0.0 ? p.smoothing * z : 0.0);
        const double slope = (p.smoothing * sigmoid(z) - (1.0 - p.smoothing) * sigmoid(-z)) / pairs;
        out.margins[i] = (float)z;
        out.weights[2 * i] = (float)(slope * each[0]);
        out.weights[2 * i + 1] = (float)(-slope * each[1]);
    }
    block_sums(all);
    if (threadIdx.x == 0) out.loss[0] = pairs > 0 ? (float)(loss / pairs) : 0.0f;
}

template <class Loss>
constexpr int used_terms() { return std::is_same<Loss, PolicyLoss>::value ? 4 : 2; }

template <class Loss>
__global__ void __launch_bounds__(kBlock) loss_chunks(const Loss p, int64_t chunks, double* slots) {
    const int64_t chunk = (int64_t)blockIdx.x * kWaves + threadIdx.x / 64;
    if (chunk < chunks) chunk_sums(p, chunk, slots);
}

template <class Loss>
__global__ void __launch_bounds__(kBlock) loss_sequences(const Loss p, const double* slots, double* sums) {
    const int i = blockIdx.x * kWaves + threadIdx.x / 64;
    if (i >= p.s.S) return;
    double v[kTerms];
    sequence_sums<used_terms<Loss>()>(p.s, i, slots, v);
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < kTerms; ++k) sums[(int64_t)i * kTerms + k] = v[k];
}

template <class Loss, class... Out>
__global__ void __launch_bounds__(kFinish) loss_finish(const Loss p, const double* sums, Out... out) {
    finish(p, sums, out...);
}

template <class Loss, class... Out>
__global__ void __launch_bounds__(kFinish) loss_at_once(const Loss p, int64_t chunks, double* slots, double* sums, Out... out) {
    const int wave = threadIdx.x / 64;
    for (int64_t c = wave; c < chunks; c += kFinish / 64) chunk_sums(p, c, slots);
    __syncthreads();
    for (int i = wave; i < p.s.S; i += kFinish / 64) {
        double v[kTerms];
        sequence_sums<used_terms<Loss>()>(p.s, i, slots, v);
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < kTerms; ++k) sums[(int64_t)i * kTerms + k] = v[k];
    }
    __syncthreads();
    finish(p, sums, out...);
}

template <class Loss, class... Out>
int loss_launch(const Loss& p, void* workspace, hipStream_t stream, Out... out) {
    const int64_t chunks = (p.s.T + kChunk - 1) / kChunk;
    double* slots = static_cast<double*>(workspace);
    double* sums = slots + (chunks + p.s.S) * kTerms;
    if (p.s.T <= one_launch_tokens<Loss>() && p.s.S <= kOneLaunchSequences) {
        hipLaunchKernelGGL((loss_at_once<Loss, Out...>), dim3(1), dim3(kFinish), 0, stream, p, chunks, slots, sums, out...);
        return launch_status();
    }
    int rc = SDGP_OK;
    if (p.s.S > 0 && chunks > 0) {
        hipLaunchKernelGGL((loss_chunks<Loss>), dim3((unsigned)((chunks + kWaves - 1) / kWaves)), dim3(kBlock), 0, stream, p, chunks, slots);
        rc = launch_status();
        if (rc != SDGP_OK) return rc;
    }
    if (p.s.S > 0) {                                                    // (a launch has workgroups)
        hipLaunchKernelGGL((loss_sequences<Loss>), dim3((unsigned)((p.s.S + kWaves - 1) / kWaves)), dim3(kBlock), 0, stream, p, slots, sums);
        rc = launch_status();
        if (rc != SDGP_OK) return rc;
    }
    hipLaunchKernelGGL((loss_finish<Loss, Out...>), dim3(1), dim3(kFinish), 0, stream, p, sums, out...);
    return launch_status();
}

// Gradients: a wavefront a chunk, 0 for tokens that do not count.
template <class Loss>
__global__ void __launch_bounds__(kBlock) loss_gradient(const Loss p, int64_t chunks, const float* g, const float* weights, float* dlogp) {
    const Sequences& s = p.s;
    const int64_t chunk = (int64_t)blockIdx.x * kWaves + threadIdx.x / 64;
    if (chunk >= chunks) return;
    const int lane = threadIdx.x & 63;
    const int64_t begin = chunk * kChunk, end = begin + kChunk < s.T ? begin + kChunk : s.T, at = begin + 4 * lane;
    Four f;
    TokenTerms t[4];
    if constexpr (std::is_same<Loss, PolicyLoss>::value) {
        f = load_tokens(p, at);
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = token_terms(p, f.logp[k], f.old[k], f.ref[k]);
    } else {
        load_mask(s, at, f.on);
    }
    const float by = g[0];
    float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int i = sequence_behind(s, begin); i < s.S; ++i) {
        const Span span = span_of(s, i);
        if (span.begin >= end) break;
        const float w = weights[i] * by;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (!(f.on[k] && at + k >= span.begin && at + k < span.end)) continue;
            if constexpr (std::is_same<Loss, PolicyLoss>::value)
                d[k] = w * policy_terms(p, t[k], p.each ? f.adv[k] : p.advantages[i]).slope;
            else d[k] = w;
        }
    }
    RowVec<SDGP_F32> r;
    r.set(d);
    if (at < s.T) store_row<SDGP_F32>(dlogp + at, 0, (int)(s.T - at < 4 ? s.T - at : 4), r);
}

template <class Loss>
int gradient_launch(const Loss& p, const float* g, const float* weights, float* dlogp, hipStream_t stream) {
    const int64_t chunks = (p.s.T + kChunk - 1) / kChunk;
    hipLaunchKernelGGL((loss_gradient<Loss>), dim3((unsigned)((chunks + kWaves - 1) / kWaves)), dim3(kBlock), 0, stream, p, chunks, g, weights,
                       dlogp);
    return launch_status();
}

}  // namespace

size_t sequence_loss_workspace(int64_t T, int64_t S) {
    return (size_t)((T + kChunk - 1) / kChunk + 2 * S) * kTerms * sizeof(double);
}

int policy_loss_launch(const PolicyLoss& p, float* out, float* weights, void* workspace, hipStream_t stream) {
    return loss_launch(p, workspace, stream, out, weights);
}

int policy_loss_bwd_launch(const PolicyLoss& p, const float* g, const float* weights, float* dlogp, hipStream_t stream) {
    return gradient_launch(p, g, weights, dlogp, stream);
}

int preference_loss_launch(const PreferenceLoss& p, float* loss, float* margins, float* weights, void* workspace, hipStream_t stream) {
    return loss_launch(p, workspace, stream, PreferenceOut{loss, margins, weights});
}

int preference_loss_bwd_launch(const Sequences& s, const float* g, const float* weights, float* dlogp, hipStream_t stream) {
    PreferenceLoss p = {};
    p.s = s;
    return gradient_launch(p, g, weights, dlogp, stream);
}

}  // namespace sdgp
