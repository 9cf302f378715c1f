// Attention forward: o = softmax(scale q k^T) v over the keys that a query sees, and lse = ln of the softmax's sum.
//
// One pass over the keys.  The scores are computed transposed, S^T = K Q^T on 32x32 tiles, so that a lane holds sixteen keys of
// one query: the running maximum m and sum l are one number a lane, and exp2(c s - c m) stands in the registers as the
// next product's operand already, O^T = V^T P^T, the keys in the order in which the lane holds them (V's columns are read
// in that order by the transposing LDS reads).  m is a bound that need not be the maximum: it moves only when a score
// passes it by 2^8, so most tiles rescale nothing.  bf16 probabilities are rounded to the nearest, as they are the operand of
// a bf16 product; their sum is taken of the unrounded ones.
#pragma once

#include "attention.h"

namespace sdgp {

// FEW: a workgroup's wavefronts share 32 rows (single tokens): two halves of the keys, each for two halves of a head's values, so that
// two workgroups fit a CU and one's loads fly while the other begins or ends.  Else each wavefront has 32 rows of its own.
template <int DT, int DC, bool FEW>
struct AttentionFwd {
    static constexpr int kWaves = 4, kThreads = 64 * kWaves;
    static constexpr int kRows = FEW ? 32 : 32 * kWaves;
    static constexpr int kSplit = 2;                                   // FEW: of the keys
    static constexpr int kKeys = FEW ? 32 * kSplit : (DT == SDGP_BF16 ? 64 : 32);
    static constexpr int kBlocks = FEW ? 1 : kKeys / 32;               // of 32 keys, a wavefront
    using T = Tile<DT, DC>;
    static constexpr int kTile = kKeys * T::kRow, kBuffer = 2 * kTile, kLds = 2 * kBuffer;
};

// Wavefronts a SIMD, as LDS and registers allow.
constexpr int attention_fwd_waves(int dt, int dc) { return dt == SDGP_F32 && dc > 64 ? 1 : 2; }

__device__ __forceinline__ float log2_sum(float mc, float l) { return (mc + __builtin_amdgcn_logf(l)) * 0.693147180559945309f; }

template <int DT, int DC, bool FEW, bool FAST>
__global__ void __launch_bounds__(256, attention_fwd_waves(DT, DC)) attention_fwd_kernel(const Attention a) {
    using L = AttentionFwd<DT, DC, FEW>;
    using T = typename L::T;
    constexpr int SIZE = Operand<DT>::kSize, STEPS = DC / 16, DB = DC / 32, NB = L::kBlocks;
    __shared__ __attribute__((aligned(512))) char lds_bytes[L::kLds];
    __shared__ float lds_ml[FEW ? 2 * 32 * L::kSplit : 1];
    SDGP_SHARED char* lds = (SDGP_SHARED char*)lds_bytes;

    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const int head = blockIdx.x % a.Hk, rest = blockIdx.x / a.Hk;       // a head's tiles on one die, whose cache holds its keys
    const int part = rest % a.parts;
    Sequence s;
    int tile, tiles;
    if (!find_tile<false, L::kRows>(a, rest / a.parts, s, tile, tiles)) return;
    tile = tiles - 1 - tile;                                            // the longest rows first
    const int row0 = tile * L::kRows, rows = s.nq * a.G;

    // This lane's query and how many keys it and its neighbours see.
    const int first_row = row0 + (FEW ? 0 : 32 * wave), row = first_row + (lane & 31);
    const auto seen = [&](int r) {                                      // by row r of the sequence
        if (r >= rows) return 0;
        return a.causal ? clamp_int((int)divide((uint32_t)r, a.by_group) + 1 + s.nk - s.nq, 0, s.nk) : s.nk;
    };
    const int mine = seen(row), fewest = seen(first_row);
    const int last = rows - 1 < row0 + L::kRows - 1 ? rows - 1 : row0 + L::kRows - 1;
    const int most = seen(last);                                        // of the workgroup
    const int most_mine = FEW ? most : seen(last < first_row + 31 ? last : first_row + 31);   // of the wavefront (rows in front of last)
    const bool any_row = first_row < rows;
    const int split = FEW ? wave % L::kSplit : 0, side = FEW ? wave / L::kSplit : 0;   // FEW: whose keys, and which blocks of values

    const int t = row < rows ? (int)divide((uint32_t)row, a.by_group) : 0, g = row < rows ? row - t * a.G : 0;
    const int64_t out_row = (int64_t)(s.q0 + t) * a.H + head * a.G + g;
    Operand<DT> q[STEPS];
    {
        const char* p = static_cast<const char*>(a.q) + ((int64_t)(s.q0 + t) * a.q_token + (int64_t)(head * a.G + g) * a.q_head) * SIZE;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) q[i] = load_operand<DT, FAST>(p, 16 * i + 8 * half, row < rows ? a.D : 0);
    }
    const char* keys = static_cast<const char*>(a.k) + ((int64_t)s.k0 * a.k_token + (int64_t)head * a.k_head) * SIZE;
    const char* values = static_cast<const char*>(a.v) + ((int64_t)s.k0 * a.v_token + (int64_t)head * a.v_head) * SIZE;
    const int64_t k_row = a.k_token * SIZE, v_row = a.v_token * SIZE;

    // This part's tiles of keys.
    const int all = (most + L::kKeys - 1) / L::kKeys, per = (all + a.parts - 1) / a.parts;
    const int begin = part * per < all ? part * per : all, end = begin + per < all ? begin + per : all;

    Feed<DT, DC, L::kKeys, FAST> fk(keys, k_row, a.D), fv(values, v_row, a.D);
    attn_f32x16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    float m = -INFINITY, l = 0.0f;
    const float slack = 8.0f / a.c;
    const auto buffer = [&](int n) { return lds + (n & 1) * L::kBuffer; };
    const auto start = [&](int n) {
        fk.start(buffer(n), n * L::kKeys, s.nk);
        fv.start(buffer(n) + L::kTile, n * L::kKeys, s.nk);
    };
    const auto finish = [&](int n) {
        fk.finish(buffer(n));
        fv.finish(buffer(n) + L::kTile);
        __syncthreads();
    };
    if (begin < end) {
        start(begin);
        finish(begin);
    }
    for (int n = begin; n < end; ++n) {
        SDGP_SHARED char *kt = buffer(n), *vt = kt + L::kTile;
        if (n + 1 < end) start(n + 1);
        const int key0 = n * L::kKeys + 32 * split;
        if (key0 < most_mine && any_row) {
            const uint32_t k_at = T::rows_lane(kt, lane), v_at = T::columns_lane(vt, lane);
            attn_f32x16 x[NB];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int r0 = 32 * (FEW ? split : b);
#pragma unroll
                for (int i = 0; i < 16; ++i) x[b][i] = 0.0f;
#pragma unroll
                for (int i = 0; i < STEPS; ++i) x[b] = multiply(T::rows(k_at, r0, i), q[i], x[b]);
            }
            if (key0 + 32 * NB > fewest) {                                  // some row does not see all of these
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (key0 + 32 * b + result_row(i, half) >= mine) x[b][i] = -INFINITY;
            }
            float top = x[0][0];
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, x[b][i]);
            top = halves_max(top);
            if (__any(top > m + slack)) {                                   // (true where m is -inf and a key is seen)
                const float now = fmaxf(m, top);
                const float factor = now == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - now) * a.c);
                m = now;
                l *= factor;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] *= factor;
            }
            const float mc = m == -INFINITY ? 0.0f : m * a.c;
            Operand<DT> p[NB][2];
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float y[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        y[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][8 * u + i], a.c, -mc));
                        l += y[i];
                    }
                    p[b][u].set(y);
                }
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                if (FEW && d % 2 != side) continue;
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int u = 0; u < 2; ++u) o[d] = multiply(T::columns(v_at, 32 * (FEW ? split : b) + 16 * u, d), p[b][u], o[d]);
            }
        }
        if (n + 1 < end) finish(n + 1);
    }
    l = halves_sum(l);
    float mc = m == -INFINITY ? 0.0f : m * a.c;

    if constexpr (FEW) {
        // The wavefronts' sums over their keys, brought to one maximum and added up.
        __syncthreads();
        float* ml = lds_ml;
        if (half == 0 && side == 0) ml[split * 32 + lane] = l != 0.0f ? mc : -INFINITY;
        __syncthreads();
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < L::kSplit; ++w) top = fmaxf(top, ml[w * 32 + (lane & 31)]);
        const float factor = l != 0.0f ? __builtin_amdgcn_exp2f(mc - top) : 0.0f;
        if (half == 0 && side == 0) ml[(L::kSplit + split) * 32 + lane] = l * factor;
        SDGP_SHARED float* sums = (SDGP_SHARED float*)lds;             // [kSplit, 32, DC]
#pragma unroll
        for (int d = 0; d < DB; ++d)
            if (d % 2 == side)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    sums[(split * 32 + (lane & 31)) * DC + ((32 * d + result_row(i, half)) ^ (lane & 31))] = o[d][i] * factor;
        __syncthreads();
        for (int e = threadIdx.x; e < 32 * DC; e += L::kThreads) {
            const int r = e / DC, d = e % DC, at = row0 + r;
            if (at >= rows || d >= a.D) continue;
            float sum = 0.0f, total = 0.0f, big = -INFINITY;
#pragma unroll
            for (int w = 0; w < L::kSplit; ++w) {
                sum += sums[(w * 32 + r) * DC + (d ^ r)];
                total += ml[(L::kSplit + w) * 32 + r];
                big = fmaxf(big, ml[w * 32 + r]);
            }
            const int tok = (int)divide((uint32_t)at, a.by_group);
            const int64_t to = (int64_t)(s.q0 + tok) * a.H + head * a.G + (at - tok * a.G);
            if (a.parts > 1) {
                const int64_t slot = (int64_t)part * ((int64_t)a.Tq * a.H) + to;
                a.part_o[slot * a.D + d] = sum;
                if (d == 0) a.part_ml[2 * slot] = big, a.part_ml[2 * slot + 1] = total;
            } else {
                const float y = total != 0.0f ? sum / total : 0.0f;
                if constexpr (DT == SDGP_BF16) static_cast<uint16_t*>(a.o)[to * a.D + d] = (uint16_t)float_to_bf16(y);
                else static_cast<float*>(a.o)[to * a.D + d] = y;
                if (d == 0) a.lse[to] = total != 0.0f ? log2_sum(big, total) : -INFINITY;
            }
        }
        return;
    }
    if (row >= rows) return;
    if (a.parts > 1) {
        const int64_t slot = (int64_t)part * ((int64_t)a.Tq * a.H) + out_row;
        if (half == 0) a.part_ml[2 * slot] = l != 0.0f ? mc : -INFINITY, a.part_ml[2 * slot + 1] = l;
#pragma unroll
        for (int d = 0; d < DB; ++d) store_block<SDGP_F32, FAST>(reinterpret_cast<char*>(a.part_o + slot * a.D), o[d], d, half, a.D, 1.0f);
        return;
    }
    const float inverse = l != 0.0f ? 1.0f / l : 0.0f;
    if (half == 0) a.lse[out_row] = l != 0.0f ? log2_sum(mc, l) : -INFINITY;
#pragma unroll
    for (int d = 0; d < DB; ++d) store_block<DT, FAST>(static_cast<char*>(a.o) + out_row * a.D * SIZE, o[d], d, half, a.D, inverse);
}

// Rows whose keys were taken in parts: one wavefront a row.  Parts without keys hold nothing: what is read of them is not used.
template <int DT>
__global__ void __launch_bounds__(256) attention_join(const Attention a) {
    const int64_t rows = (int64_t)a.Tq * a.H, r = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
    const int lane = threadIdx.x & 63;
    if (r >= rows) return;
    // up to 64 parts: one a lane
    float mc = -INFINITY, l = 0.0f;
    if (lane < a.parts) mc = a.part_ml[2 * (lane * rows + r)], l = a.part_ml[2 * (lane * rows + r) + 1];
    float top = mc;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float factor = l != 0.0f ? __builtin_amdgcn_exp2f(mc - top) : 0.0f;
    float total = l * factor;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) total += __shfl_xor(total, o);
    const float weight = total != 0.0f ? factor / total : 0.0f;
    float y[2] = {0.0f, 0.0f};                                          // values lane and lane + 64: D <= 128
    const int64_t step = rows * a.D;
    const float* from = a.part_o + r * a.D;
    for (int p0 = 0; p0 < a.parts; p0 += 4) {
        float x[4][2];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                x[k][j] = 0.0f;
                if (p0 + k < a.parts && lane + 64 * j < a.D) x[k][j] = from[(p0 + k) * step + lane + 64 * j];
            }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float w = bits_to_float((uint32_t)__builtin_amdgcn_readlane((int)float_to_bits(weight), (p0 + k) & 63));
#pragma unroll
            for (int j = 0; j < 2; ++j) y[j] += w != 0.0f ? w * x[k][j] : 0.0f;
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int d = lane + 64 * j;
        if (d >= a.D) continue;
        if constexpr (DT == SDGP_BF16) static_cast<uint16_t*>(a.o)[r * a.D + d] = (uint16_t)float_to_bf16(y[j]);
        else static_cast<float*>(a.o)[r * a.D + d] = y[j];
    }
    if (lane == 0) a.lse[r] = total != 0.0f ? log2_sum(top, total) : -INFINITY;
}

}  // namespace sdgp
