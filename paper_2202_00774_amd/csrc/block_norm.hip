// The norms around a block, with its gate and the scaled residual, in one pass, and their gradient.
//
//   a = u * r_u,  r_u = 1/sqrt(mean(u^2) + eps)         the norm after the block
//   y = residual_scale * x + gate * (a * w_post)        stored, rounded to the tensor's type
//   t = y * r_y,  r_y = 1/sqrt(mean(y^2) + eps)         the norm before the next block, of y as stored
//   h = t * w_pre
// Gradient, from dy (of the stored y) and dh:
//   dn = dh * w_pre;  dY = dy + r_y (dn - t mean(dn t));  dx = residual_scale * dY
//   da = dY * gate * w_post;  du = r_u (da - a mean(da a))
//   dw_pre = sum_rows dh t;  dw_post = sum_rows dY gate a;  dgate = sum over a gate's rows of dY a w_post
// Everything between a load and its store is fp32.  The sums over rows have a fixed order: no atomics.
#include "common.h"

namespace sdgp {

namespace {

constexpr int kBlock = 256, kWave = 64, kWaves = kBlock / kWave;

__device__ __forceinline__ float load1(const void* p, int dt, int64_t i) {
    return dt == SDGP_BF16 ? bf16_to_float(static_cast<const uint16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}

// Stores a value and returns it as it is stored.
__device__ __forceinline__ float store1(void* p, int dt, int64_t i, float v) {
    if (dt == SDGP_BF16) {
        const uint32_t b = float_to_bf16(v);
        static_cast<uint16_t*>(p)[i] = (uint16_t)b;
        return bf16_to_float(b);
    }
    static_cast<float*>(p)[i] = v;
    return v;
}

// Sum over the workgroup, the same for every thread.
__device__ __forceinline__ float block_sum(float v, float* lds) {
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) lds[threadIdx.x / kWave] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

struct Norm {
    const void *x, *u, *gate, *w_post, *w_pre;
    void *y, *h;
    float* stats;
    int64_t rows, per_gate;   // rows that share a gate
    int D, dt, wdt;
    float residual_scale, eps;
};

__global__ void __launch_bounds__(kBlock) norm_rows(const Norm n) {
    __shared__ float lds[kWaves];
    for (int64_t r = blockIdx.x; r < n.rows; r += gridDim.x) {
    const int64_t base = r * n.D;
    const int tid = threadIdx.x;
    const void* y = n.x;
    float sq = 0.0f;
    if (n.u) {
        y = n.y;
        for (int d = tid; d < n.D; d += kBlock) {
            const float u = load1(n.u, n.dt, base + d);
            sq += u * u;
        }
        const float ru = 1.0f / sqrtf(block_sum(sq, lds) / n.D + n.eps);
        if (tid == 0) n.stats[r] = ru;
        const int64_t gbase = n.gate ? r / n.per_gate * n.D : 0;
        sq = 0.0f;
        for (int d = tid; d < n.D; d += kBlock) {
            float v = load1(n.u, n.dt, base + d) * ru;
            if (n.w_post) v *= load1(n.w_post, n.wdt, d);
            if (n.gate) v *= load1(n.gate, n.dt, gbase + d);
            v = store1(n.y, n.dt, base + d, n.residual_scale * load1(n.x, n.dt, base + d) + v);
            sq += v * v;
        }
    } else {
        for (int d = tid; d < n.D; d += kBlock) {
            const float v = load1(n.x, n.dt, base + d);
            sq += v * v;
        }
    }
    if (!n.h) continue;
    const float ry = 1.0f / sqrtf(block_sum(sq, lds) / n.D + n.eps);
    if (tid == 0) n.stats[n.rows + r] = ry;
    for (int d = tid; d < n.D; d += kBlock) {
        float v = load1(y, n.dt, base + d) * ry;      // what this thread stored itself
        if (n.w_pre) v *= load1(n.w_pre, n.wdt, d);
        store1(n.h, n.dt, base + d, v);
    }
    }
}

struct NormGrad {
    const void *dy, *dh, *y, *u, *gate, *w_post, *w_pre;
    const float* stats;
    void *dx, *du, *dgate;
    float *dw_post, *dw_pre;
    float* mean;              // [rows]: mean(dn t), for the sums over rows
    int64_t rows, per_gate, groups;
    int D, dt, wdt;
    float residual_scale;
};

__device__ __forceinline__ float weight(const void* w, int dt, int64_t i) { return w ? load1(w, dt, i) : 1.0f; }

// dY of one element, dL/dy with the norm behind it taken in.
__device__ __forceinline__ float grad_y(const NormGrad& n, int64_t i, int d, float ry, float mean) {
    float v = n.dy ? load1(n.dy, n.dt, i) : 0.0f;
    if (n.dh) {
        const float dn = load1(n.dh, n.dt, i) * weight(n.w_pre, n.wdt, d);
        v += ry * (dn - load1(n.y, n.dt, i) * ry * mean);
    }
    return v;
}

__global__ void __launch_bounds__(kBlock) norm_grad_rows(const NormGrad n) {
    __shared__ float lds[kWaves];
    for (int64_t r = blockIdx.x; r < n.rows; r += gridDim.x) {
    const int64_t base = r * n.D;
    const int tid = threadIdx.x;
    float ry = 0.0f, mean = 0.0f;
    if (n.dh) {
        ry = n.stats[n.rows + r];
        float sum = 0.0f;
        for (int d = tid; d < n.D; d += kBlock)
            sum += load1(n.dh, n.dt, base + d) * weight(n.w_pre, n.wdt, d) * (load1(n.y, n.dt, base + d) * ry);
        mean = block_sum(sum, lds) / n.D;
    }
    if (tid == 0) n.mean[r] = mean;
    float ru = 0.0f, mean_a = 0.0f;
    const int64_t gbase = n.gate ? r / n.per_gate * n.D : 0;
    if (n.u) {
        ru = n.stats[r];
        float sum = 0.0f;
        for (int d = tid; d < n.D; d += kBlock) {
            const float k = weight(n.gate, n.dt, gbase + d) * weight(n.w_post, n.wdt, d);
            sum += grad_y(n, base + d, d, ry, mean) * k * (load1(n.u, n.dt, base + d) * ru);
        }
        mean_a = block_sum(sum, lds) / n.D;
    }
    for (int d = tid; d < n.D; d += kBlock) {
        const float dY = grad_y(n, base + d, d, ry, mean);
        store1(n.dx, n.dt, base + d, n.u ? n.residual_scale * dY : dY);
        if (n.u) {
            const float k = weight(n.gate, n.dt, gbase + d) * weight(n.w_post, n.wdt, d);
            store1(n.du, n.dt, base + d, ru * (dY * k - load1(n.u, n.dt, base + d) * ru * mean_a));
        }
    }
    }
}

// Sums over rows, one thread a column.
__global__ void __launch_bounds__(kBlock) norm_grad_columns(const NormGrad n) {
    const int d = blockIdx.x * kBlock + threadIdx.x;
    if (d >= n.D) return;
    float pre = 0.0f, post = 0.0f, gate = 0.0f;
    for (int64_t r = 0; r < n.rows; ++r) {
        const int64_t i = r * n.D + d;
        const float ry = n.dh ? n.stats[n.rows + r] : 0.0f;
        if (n.dh) pre += load1(n.dh, n.dt, i) * (load1(n.y, n.dt, i) * ry);
        if (!n.u) continue;
        const float da = grad_y(n, i, d, ry, n.mean[r]) * (load1(n.u, n.dt, i) * n.stats[r]);
        const int64_t g = n.gate ? r / n.per_gate : 0;
        post += da * weight(n.gate, n.dt, g * n.D + d);
        gate += da;
        if (n.gate && (r + 1) % n.per_gate == 0) {
            store1(n.dgate, n.dt, g * n.D + d, gate * weight(n.w_post, n.wdt, d));
            gate = 0.0f;
        }
    }
    if (n.dw_pre) n.dw_pre[d] = pre;
    if (n.dw_post) n.dw_post[d] = post;
}

__global__ void __launch_bounds__(kBlock) clear_words(uint16_t* __restrict__ p, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < n; i += (int64_t)gridDim.x * kBlock) p[i] = 0;
}

}  // namespace

int block_norm_bwd_no_rows(void* dgate, int64_t gate_elements, int dt, float* dw_post, float* dw_pre, int64_t D, hipStream_t stream) {
    const struct {
        void* p;
        int64_t halves;
    } all[] = {{dgate, gate_elements * (dt == SDGP_BF16 ? 1 : 2)}, {dw_post, 2 * D}, {dw_pre, 2 * D}};
    for (const auto& a : all) {
        if (a.p == nullptr || a.halves == 0) continue;
        const int64_t blocks = (a.halves + kBlock - 1) / kBlock;
        hipLaunchKernelGGL(clear_words, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(kBlock), 0, stream,
                           static_cast<uint16_t*>(a.p), a.halves);
        const int rc = launch_status();
        if (rc != SDGP_OK) return rc;
    }
    return SDGP_OK;
}

size_t block_norm_bwd_workspace(int64_t rows, int64_t, int64_t, int) { return (size_t)rows * 4; }

int block_norm_launch(const void* x, const void* u, const void* gate, const void* w_post, const void* w_pre, void* y, void* h,
                      float* stats, int64_t rows, int64_t D, int64_t groups, int dt, int wdt, float residual_scale, float eps,
                      hipStream_t stream) {
    const Norm n = {x, u, gate, w_post, w_pre, y, h, stats, rows, groups > 0 ? rows / groups : rows, (int)D, dt, wdt, residual_scale, eps};
    hipLaunchKernelGGL(norm_rows, dim3((unsigned)(rows < 65536 ? rows : 65536)), dim3(kBlock), 0, stream, n);
    return launch_status();
}

int block_norm_bwd_launch(const void* dy, const void* dh, const void* y, const void* u, const void* gate, const void* w_post,
                          const void* w_pre, const float* stats, void* dx, void* du, void* dgate, float* dw_post, float* dw_pre,
                          int64_t rows, int64_t D, int64_t groups, int dt, int wdt, float residual_scale, void* workspace,
                          hipStream_t stream) {
    const NormGrad n = {dy, dh, y, u, gate, w_post, w_pre, stats, dx, du, dgate, dw_post, dw_pre, static_cast<float*>(workspace), rows,
                        groups > 0 ? rows / groups : rows, groups, (int)D, dt, wdt, residual_scale};
    hipLaunchKernelGGL(norm_grad_rows, dim3((unsigned)(rows < 65536 ? rows : 65536)), dim3(kBlock), 0, stream, n);
    int rc = launch_status();
    if (rc != SDGP_OK) return rc;
    hipLaunchKernelGGL(norm_grad_columns, dim3((unsigned)((D + kBlock - 1) / kBlock)), dim3(kBlock), 0, stream, n);
    return launch_status();
}

}  // namespace sdgp
