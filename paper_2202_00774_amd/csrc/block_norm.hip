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
//
// Rows that fit the registers of a workgroup go to the kernels of block_norm_rows.h; the ones here take any width and
// read a row again for each sum.  Backward, either kind leaves sums over slabs of rows, which norm_grad_finish adds up.
#include "block_norm.h"

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

__global__ void __launch_bounds__(kBlock) norm_long_rows(const Norm n) {
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
        const float ru = rsqrtf(block_sum(sq, lds) / n.D + n.eps);
        if (tid == 0) n.stats[r] = ru;
        const int64_t gbase = n.gate ? r / n.per_gate * n.D : 0;
        sq = 0.0f;
        for (int d = tid; d < n.D; d += kBlock) {
            float v = mul_rn(load1(n.u, n.dt, base + d), ru);
            if (n.w_post) v = mul_rn(v, load1(n.w_post, n.wdt, d));
            if (n.gate) v = mul_rn(v, load1(n.gate, n.dt, gbase + d));
            v = store1(n.y, n.dt, base + d, add_rn(mul_rn(n.residual_scale, load1(n.x, n.dt, base + d)), v));
            sq += v * v;
        }
    } else {
        for (int d = tid; d < n.D; d += kBlock) {
            const float v = load1(n.x, n.dt, base + d);
            sq += v * v;
        }
    }
    if (!n.h) continue;
    const float ry = rsqrtf(block_sum(sq, lds) / n.D + n.eps);
    if (tid == 0) n.stats[n.rows + r] = ry;
    for (int d = tid; d < n.D; d += kBlock) {
        float v = load1(y, n.dt, base + d) * ry;      // what this thread stored itself
        if (n.w_pre) v *= load1(n.w_pre, n.wdt, d);
        store1(n.h, n.dt, base + d, v);
    }
    }
}

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

__global__ void __launch_bounds__(kBlock) norm_grad_long_rows(const NormGrad n, float* __restrict__ means) {
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
    if (tid == 0) means[r] = mean;
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

// The slabs' sums over rows of any width, one thread a column.
__global__ void __launch_bounds__(kBlock) norm_grad_columns(const NormGrad n, const float* __restrict__ means) {
    const int columns = (n.D + kBlock - 1) / kBlock;   // workgroups of a slab
    const int d = (int)(blockIdx.x % columns) * kBlock + threadIdx.x;
    if (d >= n.D) return;
    const int64_t slab = blockIdx.x / columns;
    const float w = weight(n.w_post, n.wdt, d);
    int64_t first, end;
    if (n.slabs.kind == kWholeGroups) {
        first = slab * n.slabs.len * n.per_gate;
        end = first + n.slabs.len * n.per_gate < n.rows ? first + n.slabs.len * n.per_gate : n.rows;
    } else {
        const int64_t gate0 = slab / n.slabs.parts * n.per_gate;
        first = gate0 + slab % n.slabs.parts * n.slabs.len;
        end = first + n.slabs.len < gate0 + n.per_gate ? first + n.slabs.len : gate0 + n.per_gate;
    }
    float pre = 0.0f, post = 0.0f, sum = 0.0f;
    for (int64_t r = first; r < end; ++r) {
        const int64_t i = r * n.D + d;
        const float ry = n.dh ? n.stats[n.rows + r] : 0.0f;
        if (n.dh) pre += load1(n.dh, n.dt, i) * (load1(n.y, n.dt, i) * ry);
        if (!n.u) continue;
        sum += grad_y(n, i, d, ry, means[r]) * (load1(n.u, n.dt, i) * n.stats[r]);
        if (n.slabs.kind == kWholeGroups && (r + 1) % n.per_gate == 0) {
            const int64_t g = (r / n.per_gate) * n.D + d;
            store1(n.dgate, n.dt, g, sum * w);
            post += sum * load1(n.gate, n.dt, g);
            sum = 0.0f;
        }
    }
    if (n.part_pre) n.part_pre[slab * n.D + d] = pre;
    if (n.part_post) n.part_post[slab * n.D + d] = n.slabs.kind == kWholeGroups ? post : sum;
}

// Adds up the slabs' sums: 32 columns a workgroup, 32 threads down each.  In kInGroup a gate's slabs are added first, to
// dgate, and the gates' sums times the gate to dw_post.  Fixed order throughout.
constexpr int kCols = 32, kDown = 32;

// Sum of v over `over` threads down a column (a power of two; threads k * over .. k * over + over - 1), in the first of them.
__device__ __forceinline__ float add_down(float v, int over, float (*lds)[kCols + 1]) {
    const int col = threadIdx.x % kCols, down = threadIdx.x / kCols;
    __syncthreads();
    lds[down][col] = v;
    for (int o = over / 2; o > 0; o /= 2) {
        __syncthreads();
        if ((down & (over - 1)) < o) lds[down][col] += lds[down + o][col];
    }
    __syncthreads();
    return lds[down][col];
}

__device__ __forceinline__ float add_slabs(const float* part, int D, int64_t first, int64_t end, int64_t step, int d) {
    float s[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    int64_t i = first;
    for (; i + 7 * step < end; i += 8 * step)
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] += part[(i + k * step) * D + d];
    for (; i < end; i += step) s[0] += part[i * D + d];
    return ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
}

// blockIdx.y: 0 for dw_pre, 1 for dw_post and dgate.
__global__ void __launch_bounds__(kCols* kDown) norm_grad_finish(const NormGrad n) {
    __shared__ float lds[kDown][kCols + 1];
    const int d = blockIdx.x * kCols + threadIdx.x % kCols, down = threadIdx.x / kCols;
    const bool in = d < n.D;
    const float* part = blockIdx.y == 0 ? n.part_pre : n.part_post;
    float* dw = blockIdx.y == 0 ? n.dw_pre : n.dw_post;
    if (part == nullptr) return;
    float sum = 0.0f;
    if (blockIdx.y == 0 || n.slabs.kind == kWholeGroups || n.gate == nullptr) {
        if (in) sum = add_slabs(part, n.D, down, n.slabs.count, kDown, d);
    } else {
        // each gate's slabs by as many threads as there are for each (at least one), then the gates
        int over = kDown;
        while (over > 1 && over * n.groups > kDown) over /= 2;
        const int64_t at_once = kDown / over, parts = n.slabs.parts;
        const float w = in ? weight(n.w_post, n.wdt, d) : 0.0f;
        for (int64_t g0 = 0; g0 < n.groups; g0 += at_once) {
            const int64_t g = g0 + down / over;
            const bool mine = in && g < n.groups;
            const float s = add_down(mine ? add_slabs(part, n.D, g * parts + (down & (over - 1)), (g + 1) * parts, over, d) : 0.0f, over, lds);
            if (!mine || (down & (over - 1)) != 0) continue;
            store1(n.dgate, n.dt, g * n.D + d, s * w);
            sum += s * load1(n.gate, n.dt, g * n.D + d);
        }
    }
    sum = add_down(sum, kDown, lds);
    if (in && down == 0 && dw != nullptr) dw[d] = sum;
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

// A slab costs its columns' sums written and read again, so it holds four rows for each that a workgroup has in hand (4099
// x 1001 fp32, both directions: 64 us with eight rows each, 57 with four), unless that leaves fewer than 256 workgroups, one a CU; nor are
// there more than a CU holds at 16 wavefronts.  Gates of up to 32 rows that are many (2048), and any that are very many
// (65536, which bounds the slabs), are finished by the slab that holds them: the gradient of 4100 x 1024 bf16 with 2050 gates 23 us, with
// slabs of their own 93; 65600 x 264 120 and 169.  (Fewer gates too: 2048 x 1024 with 1024 gates 15 and 45.  But not of many rows each
// on few columns: 32768 x 264 with 1024 gates 107 and 76, 16384 x 264 with 256 194 and 40.)
static Slabs make_slabs(int64_t rows, int64_t D, int64_t groups, int dt) {
    const RowShape shape = row_shape(D, dt);
    const int64_t at_once = shape.threads == 0 ? 1 : rows_at_once(shape.threads);
    const int64_t g = groups > 0 ? groups : 1, per_gate = rows / g;
    Slabs s;
    int64_t want = rows / (4 * at_once);
    const int64_t waves = shape.threads == 0 ? kBlock / kWave : shape.threads * at_once / kWave, most = 256 * (waves >= 16 ? 1 : 16 / waves);
    want = want < 256 ? 256 : want > most ? most : want;
    if (groups > 0 && (per_gate == 1 || (per_gate <= 32 && groups >= 2048) || groups >= 65536)) {
        s.kind = kWholeGroups;
        s.len = ((groups + want - 1) / want + at_once - 1) / at_once * at_once;
        s.parts = 1;
        s.count = (groups + s.len - 1) / s.len;
    } else {
        s.kind = kInGroup;
        int64_t parts = want / g;
        const int64_t steps = (per_gate + at_once - 1) / at_once;
        parts = parts < 1 ? 1 : parts > steps ? steps : parts;
        s.len = ((per_gate + parts - 1) / parts + at_once - 1) / at_once * at_once;
        s.parts = (per_gate + s.len - 1) / s.len;
        s.count = s.parts * g;
    }
    return s;
}

size_t block_norm_bwd_workspace(int64_t rows, int64_t D, int64_t groups, int dt) {
    const size_t sums = (size_t)make_slabs(rows, D, groups, dt).count * (size_t)D * 2 * sizeof(float);
    return sums + (row_shape(D, dt).threads == 0 ? (size_t)rows * sizeof(float) : 0);
}

int block_norm_launch(const void* x, const void* u, const void* gate, const void* w_post, const void* w_pre, void* y, void* h,
                      float* stats, int64_t rows, int64_t D, int64_t groups, int dt, int wdt, float residual_scale, float eps,
                      hipStream_t stream) {
    const Norm n = {x, u, gate, w_post, w_pre, y, h, stats, rows, groups > 0 ? rows / groups : rows, (int)D, dt, wdt, residual_scale, eps,
                    rows_aligned(D, dt, {x, u, gate}), rows_large(rows, D, dt)};
    const RowShape shape = row_shape(D, dt);
    if (shape.threads > 0)
        return dt == SDGP_BF16 ? norm_rows_launch<SDGP_BF16>(n, shape, stream) : norm_rows_launch<SDGP_F32>(n, shape, stream);
    hipLaunchKernelGGL(norm_long_rows, dim3((unsigned)(rows < 65536 ? rows : 65536)), dim3(kBlock), 0, stream, n);
    return launch_status();
}

int block_norm_bwd_launch(const void* dy, const void* dh, const void* y, const void* u, const void* gate, const void* w_post,
                          const void* w_pre, const float* stats, void* dx, void* du, void* dgate, float* dw_post, float* dw_pre,
                          int64_t rows, int64_t D, int64_t groups, int dt, int wdt, float residual_scale, void* workspace,
                          hipStream_t stream) {
    const Slabs slabs = make_slabs(rows, D, groups, dt);
    float* sums = static_cast<float*>(workspace);
    const int64_t each = slabs.count * D;
    const bool post = w_post != nullptr || (gate != nullptr && slabs.kind == kInGroup);
    const NormGrad n = {dy, dh, y, u, gate, w_post, w_pre, stats, dx, du, dgate, dw_post, dw_pre, w_pre ? sums : nullptr,
                        post ? sums + each : nullptr, rows, groups, groups > 0 ? rows / groups : rows, slabs, (int)D, dt, wdt, residual_scale,
                        rows_aligned(D, dt, {dy, dh, y, u}), rows_large(rows, D, dt)};
    const RowShape shape = row_shape(D, dt);
    int rc;
    if (shape.threads > 0) {
        rc = dt == SDGP_BF16 ? norm_grad_launch<SDGP_BF16>(n, shape, stream) : norm_grad_launch<SDGP_F32>(n, shape, stream);
    } else {
        float* means = sums + 2 * each;
        hipLaunchKernelGGL(norm_grad_long_rows, dim3((unsigned)(rows < 65536 ? rows : 65536)), dim3(kBlock), 0, stream, n, means);
        rc = launch_status();
        if (rc != SDGP_OK) return rc;
        if (n.part_pre || n.part_post || gate) {
            hipLaunchKernelGGL(norm_grad_columns, dim3((unsigned)((D + kBlock - 1) / kBlock * slabs.count)), dim3(kBlock), 0, stream, n, means);
            rc = launch_status();
        }
    }
    if (rc != SDGP_OK || (!n.part_pre && !n.part_post)) return rc;
    hipLaunchKernelGGL(norm_grad_finish, dim3((unsigned)((D + kCols - 1) / kCols), 2), dim3(kCols * kDown), 0, stream, n);
    return launch_status();
}

}  // namespace sdgp
