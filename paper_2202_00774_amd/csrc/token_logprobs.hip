// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and their gradient.
//
//   z = scale * x;  m = max x;  s = sum_j e^(z_j - scale m)
//   logp = (x_t - m) scale - ln s        entropy = ln s - (1/s) sum_j e^(z_j - scale m) (z_j - scale m)
//   dL/dx_j = scale * (g (d_jt - p_j) - h p_j (ln p_j + entropy)),  g = dL/dlogp, h = dL/dentropy
//
// One pass over a row: running maximum, sum and weighted sum (both brought to the new maximum when it grows), and the
// best `top` logits so far.  Differences to the maximum are taken before the scale is applied, so a mask of the type's
// lowest value cannot overflow into a NaN; in the weighted sum they are cut at -256 (in powers of two), where e^ is 0
// already, so that a logit of -inf adds 0 and not 0 * inf.  All sums are fp32.
#include "common.h"

namespace sdgp {

namespace {

constexpr int kBlock = 256, kWave = 64, kWaves = kBlock / kWave;
constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kFloor2 = -256.0f;   // exponents of two below this count as this: 2^-256 is 0 in fp32
constexpr int kMaxTop = 64;          // a wavefront keeps its best logits one a lane

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// max, sum of 2^(c (x - max)), sum of 2^(c (x - max)) * c (x - max)
struct Sums {
    float m, s, a;
};

__device__ __forceinline__ float exponent(float x, float m, float c) { return (x - m) * c; }

__device__ __forceinline__ Sums joined(const Sums& p, const Sums& q, float c) {
    Sums r;
    r.m = fmaxf(p.m, q.m);
    const float dp = fmaxf(exponent(p.m, r.m, c), kFloor2), dq = fmaxf(exponent(q.m, r.m, c), kFloor2);
    const float fp = exp2_hw(dp), fq = exp2_hw(dq);
    r.s = p.s * fp + q.s * fq;
    r.a = fp * (p.a + p.s * dp) + fq * (q.a + q.s * dq);
    return r;
}

template <int DT>
__device__ __forceinline__ float load_logit(const void* row, int64_t j) {
    if constexpr (DT == SDGP_BF16) return bf16_to_float(static_cast<const uint16_t*>(row)[j]);
    else return static_cast<const float*>(row)[j];
}

// The best logits a wavefront has met, lane i the i-th; equal logits in the order of their index.  Places not taken
// hold -inf and the index -1 (as unsigned the largest).
struct Best {
    float x;
    uint32_t j;
};

__device__ __forceinline__ bool better(float x, uint32_t j, float y, uint32_t k) { return x > y || (x == y && j < k); }

// Takes one logit (the same for all lanes) into the list.
__device__ __forceinline__ void insert(Best& b, float x, uint32_t j) {
    const float ux = __shfl_up(b.x, 1);
    const uint32_t uj = __shfl_up(b.j, 1);
    const bool keep = better(b.x, b.j, x, j);
    const bool up = (threadIdx.x & (kWave - 1)) != 0 && !better(ux, uj, x, j);   // the new one went in further up
    if (!keep) {
        b.x = up ? ux : x;
        b.j = up ? uj : j;
    }
}

template <int DT>
__global__ void __launch_bounds__(kBlock) logprob_rows(const void* __restrict__ logits, int64_t ld, const void* __restrict__ tokens,
                                                       int token_bits, float* __restrict__ logp, float* __restrict__ entropy,
                                                       float* __restrict__ top_logp, int64_t* __restrict__ top_ids,
                                                       float* __restrict__ stats, int64_t rows, int V, int top, float scale) {
    __shared__ Sums part[kWaves];
    __shared__ Best lists[kWaves][kMaxTop];
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const char* row = static_cast<const char*>(logits) + r * ld * (DT == SDGP_BF16 ? 2 : 4);
    const float c = scale * kLog2e;
    Sums t = {kLowest, 0.0f, 0.0f};
    Best best = {-INFINITY, 0xFFFFFFFFu};
    for (int j0 = 0; j0 < V; j0 += kBlock) {
        const int j = j0 + tid;
        const float x = j < V ? load_logit<DT>(row, j) : -INFINITY;
        if (x > t.m) {
            const float d = fmaxf(exponent(t.m, x, c), kFloor2), f = exp2_hw(d);
            t.a = f * (t.a + t.s * d);
            t.s *= f;
            t.m = x;
        }
        const float d = exponent(x, t.m, c), e = exp2_hw(d);
        t.s += e;
        t.a += e * fmaxf(d, kFloor2);
        if (top > 0) {
            uint64_t some = __ballot(x > __shfl(best.x, top - 1));
            while (some) {
                const int from = __builtin_ctzll(some);
                some &= some - 1;
                insert(best, __shfl(x, from), (uint32_t)(j0 + wave * kWave + from));
            }
        }
    }
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) t = joined(t, {__shfl_xor(t.m, o), __shfl_xor(t.s, o), __shfl_xor(t.a, o)}, c);

    __syncthreads();   // the first wavefront is done with the row before
    if (lane == 0) part[wave] = t;
    lists[wave][lane] = best;
    __syncthreads();
    if (wave != 0) continue;
    for (int w = 1; w < kWaves; ++w) {
        t = joined(t, part[w], c);
        for (int i = 0; i < top; ++i) insert(best, lists[w][i].x, lists[w][i].j);
    }

    const float logs = logf(t.s);                    // of an empty row: -inf
    const bool empty = t.s == 0.0f, bad = t.s != t.s;
    if (lane == 0) {
        if (logp) {
            const int64_t token = token_bits == 64 ? static_cast<const int64_t*>(tokens)[r] : (int64_t) static_cast<const int32_t*>(tokens)[r];
            float lp = 0.0f;
            if (token >= V) lp = NAN;
            else if (token >= 0) lp = empty ? -INFINITY : (load_logit<DT>(row, token) - t.m) * scale - logs;
            logp[r] = lp;
        }
        entropy[r] = empty ? 0.0f : logs - kLn2 * t.a / t.s;
        stats[2 * r] = t.m;
        stats[2 * r + 1] = logs;
    }
    if (lane < top) {
        const bool none = bad || best.j == 0xFFFFFFFFu;
        top_ids[r * top + lane] = none ? -1 : (int64_t)best.j;
        top_logp[r * top + lane] = bad ? NAN : none ? -INFINITY : (best.x - t.m) * scale - logs;
    }
    }
}

template <int DT>
__global__ void __launch_bounds__(kBlock) logprob_grad(const void* __restrict__ logits, int64_t ld, const void* __restrict__ tokens,
                                                       int token_bits, const float* __restrict__ stats, const float* __restrict__ entropy,
                                                       const float* __restrict__ g_logp, const float* __restrict__ g_entropy,
                                                       void* __restrict__ dlogits, int64_t ld_out, int64_t rows, int V, float scale) {
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const char* row = static_cast<const char*>(logits) + r * ld * (DT == SDGP_BF16 ? 2 : 4);
    char* out = static_cast<char*>(dlogits) + r * ld_out * (DT == SDGP_BF16 ? 2 : 4);
    const float m = stats[2 * r], logs = stats[2 * r + 1];
    int64_t token = -1;
    float g = 0.0f, h = 0.0f, H = 0.0f;
    if (g_logp) {
        token = token_bits == 64 ? static_cast<const int64_t*>(tokens)[r] : (int64_t) static_cast<const int32_t*>(tokens)[r];
        g = token >= V ? NAN : token >= 0 ? g_logp[r] : 0.0f;
    }
    if (g_entropy) {
        h = g_entropy[r];
        H = entropy[r];
    }
    const bool empty = logs == -INFINITY;
    for (int j = threadIdx.x; j < V; j += kBlock) {
        const float x = load_logit<DT>(row, j);
        const float l = (x - m) * scale - logs, p = exp2_hw(l * kLog2e);
        float d = -p * (g + h * (fmaxf(l, kFloor2) + H));
        if (j == token) d += g;
        d = empty ? 0.0f : d * scale;
        if constexpr (DT == SDGP_BF16) reinterpret_cast<uint16_t*>(out)[j] = (uint16_t)float_to_bf16(d);
        else reinterpret_cast<float*>(out)[j] = d;
    }
    }
}

unsigned row_grid(int64_t rows) { return (unsigned)(rows < 65536 ? rows : 65536); }

}  // namespace

size_t token_logprobs_workspace(int64_t, int64_t, int, int) { return 0; }

int token_logprobs_launch(const void* logits, int64_t ld, const void* tokens, int token_bits, float* logp, float* entropy,
                          float* top_logp, int64_t* top_ids, float* stats, int64_t rows, int64_t V, int dt, int top, float scale,
                          void*, hipStream_t stream) {
    auto kernel = dt == SDGP_BF16 ? logprob_rows<SDGP_BF16> : logprob_rows<SDGP_F32>;
    hipLaunchKernelGGL(kernel, dim3(row_grid(rows)), dim3(kBlock), 0, stream, logits, ld, tokens, token_bits, logp, entropy, top_logp,
                       top_ids, stats, rows, (int)V, top, scale);
    return launch_status();
}

int token_logprobs_bwd_launch(const void* logits, int64_t ld, const void* tokens, int token_bits, const float* stats, const float* entropy,
                              const float* g_logp, const float* g_entropy, void* dlogits, int64_t ld_out, int64_t rows, int64_t V,
                              int dt, float scale, hipStream_t stream) {
    auto kernel = dt == SDGP_BF16 ? logprob_grad<SDGP_BF16> : logprob_grad<SDGP_F32>;
    hipLaunchKernelGGL(kernel, dim3(row_grid(rows)), dim3(kBlock), 0, stream, logits, ld, tokens, token_bits, stats, entropy, g_logp,
                       g_entropy, dlogits, ld_out, rows, (int)V, scale);
    return launch_status();
}

}  // namespace sdgp
