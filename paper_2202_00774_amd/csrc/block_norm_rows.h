// Block norms of rows that fit the registers, forward and backward (the formulas stand in block_norm.hip).
//
// Bound by memory: 8 bytes an element forward (x, u in; y, h out), 12 backward (y, u, dy, dh in; dx, du out) in bf16, with
// 25 and 34 vector instructions beside them.  Measured: 32768 x 4096 bf16 forward 202 us (5.3 TB/s), backward 280 (5.8 TB/s) and 6
// for the slabs' sums; 16384 x 2048 with 16 gates 45, 67 and 6.  Every value is loaded once and stays in registers, packed as stored,
// until its row's sums are known.  Backward, the second norm's sum depends on the first's result (dY holds the
// mean of dn t), but linearly: with v = dy + r_y dn,
//     sum dY k a = sum v k a - r_y mean(dn t) sum t k a,        k = gate w_post,
// so all three sums go over the lanes together and a row costs one exchange, not two.
#pragma once

#include "block_norm.h"

namespace sdgp {

namespace {

template <int T>
constexpr int norm_block() { return T * rows_at_once(T); }

template <int DT, int T, int NV, bool BLOCK, Caching RESULTS>
__global__ void __launch_bounds__(norm_block<T>()) norm_fwd(const Norm n, int64_t rows_per_wg) {
    using V = RowVec<DT>;
    constexpr int N = V::kN, R = norm_block<T>() / T;
    constexpr bool kTurns = RESULTS == kStream;   // large tensors: rows in turn
    constexpr int64_t kSize = sizeof(typename V::Elem);
    __shared__ float lds[row_lds<T, 1>()];
    int turn = 0;
    const int t = threadIdx.x % T, sub = threadIdx.x / T;
    // rows in turn, or a run of them
    const int64_t first = (int64_t)blockIdx.x * (kTurns ? R : rows_per_wg), step = kTurns ? (int64_t)gridDim.x * R : R;
    const int64_t end = kTurns || first + rows_per_wg > n.rows ? n.rows : first + rows_per_wg;
    const float inv_d = 1.0f / (float)n.D;

    float post[NV][N], pre[NV][N];
    V gate[NV];
    const bool many_gates = BLOCK && n.gate != nullptr && n.per_gate != n.rows;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int e = (v * T + t) * N;
        load_weights<N>(n.w_pre, n.wdt, e, n.D, pre[v]);
        if constexpr (BLOCK) {
            load_weights<N>(n.w_post, n.wdt, e, n.D, post[v]);
            if (n.gate != nullptr) gate[v] = load_row<DT>(n.gate, e, n.D);
        }
    }

    for (int64_t r0 = first; r0 < end; r0 += step) {
        const int64_t r = r0 + sub;
        const bool live = r < end;
        const int D = live ? n.D : 0;
        const int64_t at = (live ? r : first) * n.D * kSize;
        V x[NV], u[NV];
        const auto load = [&](auto caching) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int e = (v * T + t) * N;
                x[v] = load_row<DT, decltype(caching)::value>(static_cast<const char*>(n.x) + at, e, D);
                if constexpr (BLOCK) u[v] = load_row<DT, decltype(caching)::value>(static_cast<const char*>(n.u) + at, e, D);
            }
        };
        if (n.aligned) load(Cached<kStream>{});
        else load(Cached<kKeep>{});
        float sum[1];
        if constexpr (BLOCK) {
            if (many_gates) {
                const int64_t gat = (live ? r : first) / n.per_gate * n.D * kSize;
#pragma unroll
                for (int v = 0; v < NV; ++v) gate[v] = load_row<DT>(static_cast<const char*>(n.gate) + gat, (v * T + t) * N, D);
            }
            sum[0] = 0.0f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < N; ++i) sum[0] += u[v].get(i) * u[v].get(i);
            row_sums<T, 1>(sum, lds, turn);
            const float ru = rsqrtf(sum[0] * inv_d + n.eps);
            if (t == 0 && live) n.stats[r] = ru;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float y[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    // in the formula's order, one rounding each: y is rounded again as it is stored, and all that follows
                    // is computed from that
                    float a = mul_rn(mul_rn(u[v].get(i), ru), post[v][i]);
                    if (n.gate != nullptr) a = mul_rn(gate[v].get(i), a);
                    y[i] = add_rn(mul_rn(n.residual_scale, x[v].get(i)), a);
                }
                x[v].set(y);   // y from here on, rounded as it is stored
                store_row<DT, RESULTS>(static_cast<char*>(n.y) + at, (v * T + t) * N, D, x[v]);
            }
            if (n.h == nullptr) continue;
        }
        sum[0] = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < N; ++i) sum[0] += x[v].get(i) * x[v].get(i);
        row_sums<T, 1>(sum, lds, turn);
        const float ry = rsqrtf(sum[0] * inv_d + n.eps);
        if (t == 0 && live) n.stats[n.rows + r] = ry;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float h[N];
#pragma unroll
            for (int i = 0; i < N; ++i) h[i] = x[v].get(i) * ry * pre[v][i];
            V q;
            q.set(h);
            store_row<DT, RESULTS>(static_cast<char*>(n.h) + at, (v * T + t) * N, D, q);
        }
    }
}

// What the gradient of one row reads.
template <int DT, int NV>
struct Row {
    RowVec<DT> y[NV], u[NV], dy[NV], dh[NV];
    float ry, ru;
};

template <Caching CACHING, int T, bool BLOCK, int DT, int NV>
__device__ __forceinline__ void load_as(Row<DT, NV>& row, const NormGrad& n, int64_t r, int64_t end, int t) {
    constexpr int N = RowVec<DT>::kN;
    const bool live = r < end;
    const int D = live ? n.D : 0, Dh = n.dh != nullptr ? D : 0;
    const int64_t at = live ? r * n.D * (int64_t)sizeof(typename RowVec<DT>::Elem) : 0;
    row.ry = Dh > 0 ? n.stats[n.rows + r] : 0.0f;
    row.ru = BLOCK && live ? n.stats[r] : 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int e = (v * T + t) * N;
        row.y[v] = load_row<DT, CACHING>(static_cast<const char*>(n.y) + at, e, Dh);
        row.dh[v] = load_row<DT, CACHING>(static_cast<const char*>(n.dh) + at, e, Dh);
        row.dy[v] = load_row<DT, CACHING>(static_cast<const char*>(n.dy) + at, e, n.dy != nullptr ? D : 0);
        if constexpr (BLOCK) row.u[v] = load_row<DT, CACHING>(static_cast<const char*>(n.u) + at, e, D);
    }
}

template <int T, bool BLOCK, int DT, int NV>
__device__ __forceinline__ void load(Row<DT, NV>& row, const NormGrad& n, int64_t r, int64_t end, int t) {
    if (n.aligned) load_as<kStream, T, BLOCK>(row, n, r, end, t);
    else load_as<kKeep, T, BLOCK>(row, n, r, end, t);
}

// MODE: kNoBlock, or how the slab is cut; kRowGates: whole groups of one row each, whose gate's gradient needs no sum
// (4099 x 1001 fp32 57.3 us, 58.5 as kWholeGroups; 4096 x 8192 bf16 197 and 219, both directions).
constexpr int kNoBlock = 2, kRowGates = 3;

template <int DT, int T, int NV, int MODE, Caching RESULTS>
__global__ void __launch_bounds__(norm_block<T>()) norm_bwd(const NormGrad n) {
    using V = RowVec<DT>;
    constexpr int N = V::kN, R = norm_block<T>() / T, kColumns = T * NV * N;
    constexpr bool BLOCK = MODE != kNoBlock, kWhole = MODE == kWholeGroups || MODE == kRowGates, kTurns = RESULTS == kStream;
    constexpr int64_t kSize = sizeof(typename V::Elem);
    __shared__ float lds[R > 1 ? R * kColumns : row_lds<T, 3>()];
    int turn = 0;
    const int t = threadIdx.x % T, sub = threadIdx.x / T;
    const float inv_d = 1.0f / (float)n.D;

    // Weights stay in registers, k = gate * w_post with them; but with two vectors a thread, of 1024 with 128 registers
    // each, they are read again for every row (in registers they spilled 300).  The next row is not asked for ahead of its
    // turn: that takes 25 registers, and a third or fourth wavefront a SIMD hides more (16384 x 2048: 134 us, without 124).
    constexpr bool kHeld = NV == 1;
    // Where gates are many a gate stays as it is stored, beside w_post, and k is computed for every row, so that nothing waits
    // for the gate before the row's loads are on their way (20000 x 1001 fp32, a gate a row, both directions: 266 us without, 240 with
    // it).  With 1024 threads, of 128 registers each, k is computed beforehand (4096 x 8192 bf16, a gate a row, 197 us either way; the gradient
    // of 16400 x 8000 with eight rows a gate 491, as stored 497; with a gate a row 4100 x 8000 184, as stored 164).
    constexpr bool kRaw = kHeld && T < 1024 && kWhole;
    float w_pre[NV][N], k[NV][N];   // k: w_post where kRaw
    V gates[NV];
    float sum_pre[NV][N], sum_post[NV][N];  // dh t, and dY a (kInGroup) or dY gate a (kWholeGroups)
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        if constexpr (kHeld) load_weights<N>(n.w_pre, n.wdt, (v * T + t) * N, n.D, w_pre[v]);
        if constexpr (kRaw) load_weights<N>(n.w_post, n.wdt, (v * T + t) * N, n.D, k[v]);
#pragma unroll
        for (int i = 0; i < N; ++i) sum_pre[v][i] = 0.0f, sum_post[v][i] = 0.0f;
    }

    // the gates of this slab: one (kInGroup), or `len` of them, each sub-group of threads taking its own
    const int64_t gate0 = kWhole ? (int64_t)blockIdx.x * n.slabs.len : (int64_t)blockIdx.x / n.slabs.parts;
    const int64_t gate1 = !kWhole ? gate0 + 1 : gate0 + n.slabs.len < n.groups ? gate0 + n.slabs.len : n.groups;
    for (int64_t q0 = gate0; q0 < gate1; q0 += kWhole ? R : 1) {
        const int64_t q = kWhole ? q0 + sub : q0;
        const bool mine = q < gate1;
        const int Dg = mine ? n.D : 0;   // threads without a gate hold zeros, not another's: 0 times its infinities is a NaN
        const char* gate_row = static_cast<const char*>(n.gate) + (mine ? q : gate0) * n.D * kSize;
        const auto gated = [&](int e, float (&kv)[N]) {
            load_weights<N>(n.w_post, n.wdt, e, n.D, kv);
            if (n.gate == nullptr) return;
            const V g = load_row<DT>(gate_row, e, Dg);
#pragma unroll
            for (int i = 0; i < N; ++i) kv[i] *= g.get(i);
        };
        float sum_gate[NV][N];
        if constexpr (BLOCK) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if constexpr (kRaw) gates[v] = load_row<DT>(gate_row, (v * T + t) * N, Dg);
                else if constexpr (kHeld) gated((v * T + t) * N, k[v]);
#pragma unroll
                for (int i = 0; i < N; ++i) sum_gate[v][i] = 0.0f;
            }
        }
        const auto weights = [&](int v, float (&wv)[N], float (&kv)[N]) {
            if constexpr (kHeld) {
#pragma unroll
                for (int i = 0; i < N; ++i) wv[i] = w_pre[v][i], kv[i] = kRaw ? k[v][i] * gates[v].get(i) : BLOCK ? k[v][i] : 0.0f;
            } else {
                int e = (v * T + t) * N;
                asm volatile("" : "+v"(e));   // in every row anew, not once in front of them
                load_weights<N>(n.w_pre, n.wdt, e, n.D, wv);
                if constexpr (BLOCK) gated(e, kv);
            }
        };
        int64_t first = q * n.per_gate, end = first + n.per_gate;
        if constexpr (!kWhole) {
            first += (int64_t)(blockIdx.x - gate0 * n.slabs.parts) * (kTurns ? R : n.slabs.len);
            if (!kTurns && first + n.slabs.len < end) end = first + n.slabs.len;
        }
        const int64_t rows = MODE == kRowGates ? 1 : kWhole ? n.per_gate : end - first;   // the same for all threads
        const int64_t step = kWhole ? 1 : kTurns ? R * n.slabs.parts : R;
        for (int64_t i0 = 0; i0 < rows; i0 += step) {
            const int64_t r = first + i0 + (kWhole ? 0 : sub);
            const int D = mine && r < end ? n.D : 0;
            const int64_t at = D > 0 ? r * n.D * kSize : 0;
            Row<DT, NV> row;
            load<T, BLOCK>(row, n, r, mine ? end : 0, t);
            const auto &y = row.y, &u = row.u, &dy = row.dy, &dh = row.dh;
            const float ry = row.ry, ru = row.ru;
            float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float wv[N], kv[N];
                weights(v, wv, kv);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float dn = dh[v].get(i) * wv[i], tt = y[v].get(i) * ry;
                    s[0] += dn * tt;
                    if constexpr (BLOCK) {
                        const float ka = kv[i] * (u[v].get(i) * ru);
                        s[1] += ka * (dy[v].get(i) + ry * dn);
                        s[2] += ka * tt;
                    }
                }
            }
            if constexpr (BLOCK) {
                row_sums<T, 3>(s, lds, turn);
            } else {
                float one[1] = {s[0]};
                row_sums<T, 1>(one, lds, turn);
                s[0] = one[0];
            }
            const float c = ry * (s[0] * inv_d);              // r_y mean(dn t)
            const float mean_a = (s[1] - c * s[2]) * inv_d;   // mean(dY k a)
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int e = (v * T + t) * N;
                float dx[N], du[N], wv[N], kv[N];
                weights(v, wv, kv);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float g = dh[v].get(i), tt = y[v].get(i) * ry;
                    const float dY = dy[v].get(i) + ry * (g * wv[i]) - c * tt;
                    sum_pre[v][i] += g * tt;
                    dx[i] = dY;
                    if constexpr (BLOCK) {
                        const float a = u[v].get(i) * ru, da = dY * a;
                        dx[i] = n.residual_scale * dY;
                        du[i] = ru * (dY * kv[i] - a * mean_a);
                        if constexpr (kWhole) sum_gate[v][i] += da;
                        else sum_post[v][i] += da;
                    }
                }
                V o;
                o.set(dx);
                store_row<DT, RESULTS>(static_cast<char*>(n.dx) + at, e, D, o);
                if constexpr (BLOCK) {
                    o.set(du);
                    store_row<DT, RESULTS>(static_cast<char*>(n.du) + at, e, D, o);
                }
            }
        }
        if constexpr (kWhole) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int e = (v * T + t) * N;
                float w[N], d[N];
                V g;
                if constexpr (kRaw) {
                    g = gates[v];
#pragma unroll
                    for (int i = 0; i < N; ++i) w[i] = k[v][i];
                } else {
                    load_weights<N>(n.w_post, n.wdt, e, n.D, w);
                    g = load_row<DT>(gate_row, e, Dg);
                }
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    d[i] = sum_gate[v][i] * w[i];
                    sum_post[v][i] += sum_gate[v][i] * g.get(i);
                }
                V o;
                o.set(d);
                store_row<DT>(static_cast<char*>(n.dgate) + (mine ? q : gate0) * n.D * kSize, e, mine ? n.D : 0, o);
            }
        }
    }

    // the slab's sums, those of its sub-groups of threads added up in their order
    const auto leave = [&](float* part, const float (&sum)[NV][N]) {
        if (part == nullptr) return;
        part += (int64_t)blockIdx.x * n.D;
        if constexpr (R > 1) {
            __syncthreads();
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < N; ++i) lds[sub * kColumns + (v * T + t) * N + i] = sum[v][i];
            __syncthreads();
            for (int d = threadIdx.x; d < n.D; d += norm_block<T>()) {
                float s = 0.0f;
                for (int g = 0; g < R; ++g) s += lds[g * kColumns + d];
                part[d] = s;
            }
        } else {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < N; i += 4) {
                    RowVec<SDGP_F32> o;
                    const float f[4] = {sum[v][i], sum[v][i + 1], sum[v][i + 2], sum[v][i + 3]};
                    o.set(f);
                    store_row<SDGP_F32>(part, (v * T + t) * N + i, n.D, o);
                }
        }
    };
    leave(n.part_pre, sum_pre);
    if constexpr (BLOCK) leave(n.part_post, sum_post);
}

}  // namespace

template <int DT>
int norm_rows_launch(const Norm& n, RowShape shape, hipStream_t stream) {
    const int R = rows_at_once(shape.threads);
    // workgroups that are there at once, about; each keeps the weights in registers over its rows
    const int64_t most = shape.threads <= 256 ? 2048 : shape.threads <= 512 ? 1024 : 512;
    const int64_t groups = (n.rows + R - 1) / R, per = (groups + most - 1) / most * R;
    const dim3 grid((unsigned)((n.rows + per - 1) / per)), block(shape.threads * rows_at_once(shape.threads));
#define SDGP_CASE(T, NV)                                                                                              \
    if (shape.threads == T && shape.vecs == NV) {                                                                     \
        auto kernel = n.u != nullptr ? (n.large ? norm_fwd<DT, T, NV, true, kStream> : norm_fwd<DT, T, NV, true, kKeep>)     \
                                     : (n.large ? norm_fwd<DT, T, NV, false, kStream> : norm_fwd<DT, T, NV, false, kKeep>);  \
        hipLaunchKernelGGL(kernel, grid, block, 0, stream, n, per);                                                   \
        return launch_status();                                                                                       \
    }
    SDGP_CASE(16, 1) SDGP_CASE(32, 1) SDGP_CASE(64, 1) SDGP_CASE(128, 1) SDGP_CASE(192, 1) SDGP_CASE(256, 1) SDGP_CASE(384, 1)
    SDGP_CASE(512, 1) SDGP_CASE(768, 1) SDGP_CASE(1024, 1) SDGP_CASE(1024, 2)
#undef SDGP_CASE
    return SDGP_ERR_SHAPE;
}

template <int DT>
int norm_grad_launch(const NormGrad& n, RowShape shape, hipStream_t stream) {
    const dim3 grid((unsigned)n.slabs.count), block(shape.threads * rows_at_once(shape.threads));
#define SDGP_CASE(T, NV)                                                                                              \
    if (shape.threads == T && shape.vecs == NV) {                                                                     \
        const auto pick = [&](auto results) {                                                                         \
            constexpr Caching C = decltype(results)::value;                                                           \
            return n.u == nullptr ? norm_bwd<DT, T, NV, kNoBlock, C>                                                  \
                   : n.slabs.kind == kInGroup ? norm_bwd<DT, T, NV, kInGroup, C>                                            \
                   : n.per_gate == 1 ? norm_bwd<DT, T, NV, kRowGates, C> : norm_bwd<DT, T, NV, kWholeGroups, C>;              \
        };                                                                                                            \
        hipLaunchKernelGGL((n.large ? pick(Cached<kStream>{}) : pick(Cached<kKeep>{})), grid, block, 0, stream, n);   \
        return launch_status();                                                                                       \
    }
    SDGP_CASE(16, 1) SDGP_CASE(32, 1) SDGP_CASE(64, 1) SDGP_CASE(128, 1) SDGP_CASE(192, 1) SDGP_CASE(256, 1) SDGP_CASE(384, 1)
    SDGP_CASE(512, 1) SDGP_CASE(768, 1) SDGP_CASE(1024, 1) SDGP_CASE(1024, 2)
#undef SDGP_CASE
    return SDGP_ERR_SHAPE;
}

}  // namespace sdgp
