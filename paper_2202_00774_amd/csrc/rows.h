// Rows of fp32 or bf16 values in registers: vector loads and stores at any element alignment, sums over the lanes that
// share a row.
#pragma once

#include <type_traits>

#include "common.h"

namespace sdgp {

// Sixteen bytes of a row as one load.  The address is aligned to an element only: rows of odd widths and tensors cut out
// of others start anywhere, and global memory takes such accesses (on whole lines they cost nothing extra).
template <int DT>
struct RowVec;

template <>
struct RowVec<SDGP_F32> {
    static constexpr int kN = 4;
    using Elem = float;
    float v[4];
    __device__ __forceinline__ float get(int i) const { return v[i]; }
    __device__ __forceinline__ void set(const float (&f)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = f[i];
    }
};

template <>
struct RowVec<SDGP_BF16> {
    static constexpr int kN = 8;
    using Elem = uint16_t;
    uint32_t v[4];
    __device__ __forceinline__ float get(int i) const { return bits_to_float((i & 1) ? (v[i / 2] & 0xFFFF0000u) : (v[i / 2] << 16)); }
    __device__ __forceinline__ void set(const float (&f)[8]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = float2_to_bf16x2(f[2 * i], f[2 * i + 1]);
    }
};

typedef uint32_t u32x4_half_aligned __attribute__((ext_vector_type(4), aligned(2), may_alias));
typedef uint32_t u32x4_word_aligned __attribute__((ext_vector_type(4), aligned(4), may_alias));

template <int DT>
using Unaligned16 = typename std::conditional<DT == SDGP_BF16, u32x4_half_aligned, u32x4_word_aligned>::type;

// kStream: the line is not needed again soon (a hint to the caches).  A template argument: of two stores that a flag
// chooses between, alike but for the hint, the compiler makes one without it.
enum Caching { kKeep, kStream };
template <Caching C>
using Cached = std::integral_constant<Caching, C>;

// Elements [e, e + kN) of a row of `n`; what lies outside is 0 and is not read.
template <int DT, Caching CACHING = kKeep>
__device__ __forceinline__ RowVec<DT> load_row(const void* row, int e, int n, uint32_t fill = 0u) {
    constexpr int N = RowVec<DT>::kN;
    union {
        RowVec<DT> r;
        uint32_t w[4];
        typename RowVec<DT>::Elem x[N];
    } u;
    const auto* p = static_cast<const typename RowVec<DT>::Elem*>(row) + e;
    if (e + N <= n) {
        const auto* at = reinterpret_cast<const Unaligned16<DT>*>(p);
        const auto q = CACHING == kStream ? __builtin_nontemporal_load(at) : *at;
#pragma unroll
        for (int i = 0; i < 4; ++i) u.w[i] = q[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) u.w[i] = fill;
#pragma unroll
        for (int i = 0; i < N - 1; ++i)
            if (e + i < n) u.x[i] = p[i];
    }
    return u.r;
}

template <int DT, Caching CACHING = kKeep>
__device__ __forceinline__ void store_row(void* row, int e, int n, const RowVec<DT>& r) {
    constexpr int N = RowVec<DT>::kN;
    union {
        RowVec<DT> r;
        uint32_t w[4];
        typename RowVec<DT>::Elem x[N];
    } u;
    u.r = r;
    auto* p = static_cast<typename RowVec<DT>::Elem*>(row) + e;
    if (e + N <= n) {
        Unaligned16<DT> q;
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = u.w[i];
        auto* at = reinterpret_cast<Unaligned16<DT>*>(p);
        if constexpr (CACHING == kStream) __builtin_nontemporal_store(q, at);
        else *at = q;
    } else {
#pragma unroll
        for (int i = 0; i < N - 1; ++i)
            if (e + i < n) p[i] = u.x[i];
    }
}

// kN values of a vector [n] of either type, as fp32; ones where there is none.
template <int N>
__device__ __forceinline__ void load_weights(const void* w, int dt, int e, int n, float (&f)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = 1.0f;
    if (w == nullptr) return;
    if (dt == SDGP_F32) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const auto v = load_row<SDGP_F32>(w, e + i, n);
#pragma unroll
            for (int k = 0; k < 4; ++k) f[i + k] = v.get(k);
        }
    } else if constexpr (N == 8) {
        const auto v = load_row<SDGP_BF16>(w, e, n);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = v.get(k);
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) f[k] = e + k < n ? bf16_to_float(static_cast<const uint16_t*>(w)[e + k]) : 0.0f;
    }
}

// Product and sum with a rounding each, never fused into one operation: where a result's last bit decides a later
// rounding, it should not depend on what the compiler fused.
__device__ __forceinline__ float mul_rn(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}
__device__ __forceinline__ float add_rn(float a, float b) {
#pragma clang fp contract(off)
    return a + b;
}

template <int CTRL>
__device__ __forceinline__ float lane_swap(float v) {
    return bits_to_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)float_to_bits(v), CTRL, 0xF, 0xF, true));
}

// Sum over the 16 lanes of a DPP row, in every one of them: pairs, fours, then the row mirrored in halves and whole.
__device__ __forceinline__ float sum16(float v) {
    v += lane_swap<0xB1>(v);    // quad_perm 1 0 3 2
    v += lane_swap<0x4E>(v);    // quad_perm 2 3 0 1
    v += lane_swap<0x141>(v);   // row_half_mirror
    v += lane_swap<0x140>(v);   // row_mirror
    return v;
}

__device__ __forceinline__ float lane_value(float v, int lane) {
    return bits_to_float((uint32_t)__builtin_amdgcn_readlane((int)float_to_bits(v), lane));
}

__device__ __forceinline__ float sum64(float v) {
    v = sum16(v);
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}

__device__ __forceinline__ float sum32(float v) {
    v = sum16(v);
    return v + bits_to_float((uint32_t)__builtin_amdgcn_ds_swizzle((int)float_to_bits(v), 0x401F));   // the lane 16 away
}

// Sums of K values over the T threads that share a row, the same for all of them.  Up to 64 stay inside a wavefront;
// above that the wavefronts meet in `lds` (row_lds floats), which the calls take in turn (`turn` flips), so one
// barrier a call is enough: a wavefront can be at most one call ahead of another.  All threads of the workgroup call it.
template <int T, int K>
constexpr int row_lds() { return T > 64 ? 2 * K * (T < 192 ? 4 : T / 64) : 1; }

template <int T, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float* lds, int& turn) {
    if constexpr (T == 16) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = sum16(v[k]);
    } else if constexpr (T == 32) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = sum32(v[k]);
    } else {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = sum64(v[k]);
        if constexpr (T > 64) {
            constexpr int W = T / 64, kAll = row_lds<T, K>() / (2 * K);   // wavefronts a row, a workgroup
            float* at = lds + turn * (K * kAll);
            if ((threadIdx.x & 63) == 0) {
#pragma unroll
                for (int k = 0; k < K; ++k) at[k * kAll + threadIdx.x / 64] = v[k];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float s = 0.0f;
#pragma unroll
                for (int w = 0; w < W; ++w) s += at[k * kAll + threadIdx.x / T * W + w];
                v[k] = s;
            }
            turn ^= 1;
        }
    }
}

}  // namespace sdgp
