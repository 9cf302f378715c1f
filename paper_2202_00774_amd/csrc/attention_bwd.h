// Gradients of attention, from dO, the inputs, o and lse.
//
//   P = exp(scale q k^T - lse),  delta = sum_d dO o,  dS = P (dO V^T - delta)
//   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO, the latter two summed over a key head's queries
// Two kernels without atomics: one owns queries and passes over the keys (dQ, and delta on the way), one owns keys and passes
// over the queries (dK, dV).  Each computes the scores again: 7 products of 2 D flops a pair instead of 5, for sums in
// a fixed order that are read and written once.  As forward, every 32x32 result stands in the registers as the next
// product's operand: with the owned rows in the results' columns, a lane holds sixteen of the passing rows.  P and dS are rounded
// to bf16 for bf16 tensors, as operands of bf16 products; the sums are fp32.
#pragma once

#include "attention.h"

namespace sdgp {

constexpr float kLog2E = 1.44269504088896341f;

template <int DT, int DC>
struct AttentionDq {
    static constexpr int kThreads = 256, kRows = 128, kKeys = DT == SDGP_BF16 ? 64 : 32, kBlocks = kKeys / 32;
    using T = Tile<DT, DC>;
    static constexpr int kTile = kKeys * T::kRow, kBuffer = 2 * kTile, kLds = 2 * kBuffer;
};

template <int DT, int DC>
__global__ void __launch_bounds__(256, DT == SDGP_BF16 ? 2 : 1) attention_dq_kernel(const Attention a) {
    using L = AttentionDq<DT, DC>;
    using T = typename L::T;
    constexpr int SIZE = Operand<DT>::kSize, STEPS = DC / 16, DB = DC / 32;
    __shared__ __attribute__((aligned(16))) char lds_bytes[L::kLds];
    SDGP_SHARED char* lds = (SDGP_SHARED char*)lds_bytes;

    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const int head = blockIdx.x % a.Hk;
    Sequence s;
    int tile, tiles;
    if (!find_tile<false, L::kRows>(a, blockIdx.x / a.Hk, s, tile, tiles)) return;
    tile = tiles - 1 - tile;
    const int row0 = tile * L::kRows, rows = s.nq * a.G;
    const int first_row = row0 + 32 * wave, row = first_row + (lane & 31);
    const auto seen = [&](int r) {
        if (r >= rows) return 0;
        return a.causal ? clamp_int((int)divide((uint32_t)r, a.by_group) + 1 + s.nk - s.nq, 0, s.nk) : s.nk;
    };
    const int mine = seen(row), fewest = seen(first_row);
    const int last = rows - 1 < row0 + L::kRows - 1 ? rows - 1 : row0 + L::kRows - 1;
    const int most = seen(last), most_mine = seen(last < first_row + 31 ? last : first_row + 31);
    const bool any_row = first_row < rows;

    const int t = row < rows ? (int)divide((uint32_t)row, a.by_group) : 0, g = row < rows ? row - t * a.G : 0;
    const int64_t out_row = (int64_t)(s.q0 + t) * a.H + head * a.G + g;
    const int width = row < rows ? a.D : 0;
    Operand<DT> q[STEPS], dO[STEPS];
    float delta = 0.0f;
    {
        const char* p = static_cast<const char*>(a.q) + ((int64_t)(s.q0 + t) * a.q_token + (int64_t)(head * a.G + g) * a.q_head) * SIZE;
        const char* pd = static_cast<const char*>(a.d_o) + out_row * a.D * SIZE;
        const char* po = static_cast<const char*>(a.o_in) + out_row * a.D * SIZE;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            q[i] = load_operand<DT>(p, 16 * i + 8 * half, width);
            dO[i] = load_operand<DT>(pd, 16 * i + 8 * half, width);
            const Operand<DT> o = load_operand<DT>(po, 16 * i + 8 * half, width);
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = __builtin_fmaf(dO[i].get(e), o.get(e), delta);
        }
    }
    delta = halves_sum(delta);
    const float lse2 = row < rows ? a.lse[out_row] * kLog2E : 0.0f;
    if (row < rows && half == 0) a.delta[out_row] = delta;

    const char* keys = static_cast<const char*>(a.k) + ((int64_t)s.k0 * a.k_token + (int64_t)head * a.k_head) * SIZE;
    const char* values = static_cast<const char*>(a.v) + ((int64_t)s.k0 * a.v_token + (int64_t)head * a.v_head) * SIZE;
    const int64_t k_row = a.k_token * SIZE, v_row = a.v_token * SIZE;
    const int end = (most + L::kKeys - 1) / L::kKeys;

    Stage<DT, DC, L::kKeys, L::kThreads> sk, sv;
    const auto fetch = [&](int n) {
        sk.load([&](int r) { const int at = n * L::kKeys + r; return at < s.nk ? keys + at * k_row : nullptr; }, a.D);
        sv.load([&](int r) { const int at = n * L::kKeys + r; return at < s.nk ? values + at * v_row : nullptr; }, a.D);
    };
    attn_f32x16 dq[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dq[d][i] = 0.0f;
    if (end > 0) fetch(0);
    for (int n = 0; n < end; ++n) {
        SDGP_SHARED char* kt = lds + (n & 1) * L::kBuffer;
        SDGP_SHARED char* vt = kt + L::kTile;
        sk.store(kt);
        sv.store(vt);
        __syncthreads();
        if (n + 1 < end) fetch(n + 1);
#pragma unroll
        for (int b = 0; b < L::kBlocks; ++b) {
            const int key0 = n * L::kKeys + 32 * b;
            if (key0 >= most_mine || !any_row) continue;
            attn_f32x16 x, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = dp[i] = 0.0f;
#pragma unroll
            for (int i = 0; i < STEPS; ++i) x = multiply(T::rows(kt, 32 * b, i, lane), q[i], x);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) dp = multiply(T::rows(vt, 32 * b, i, lane), dO[i], dp);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.c, -lse2)) * (dp[i] - delta);
            if (key0 + 32 > fewest) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (key0 + result_row(i, half) >= mine) x[i] = 0.0f;
            }
            Operand<DT> ds[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = x[8 * u + i];
                ds[u].set(y);
            }
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int u = 0; u < 2; ++u) dq[d] = multiply(T::columns(kt, 32 * b + 16 * u, d, lane), ds[u], dq[d]);
        }
    }
    if (row >= rows) return;
#pragma unroll
    for (int d = 0; d < DB; ++d) store_block<DT>(static_cast<char*>(a.dq) + out_row * a.D * SIZE, dq[d], d, half, a.D, a.scale);
}

template <int DT, int DC>
struct AttentionDkv {
    static constexpr int kThreads = 256, kKeys = 128, kRows = DT == SDGP_BF16 ? 64 : 32, kBlocks = kRows / 32;
    using T = Tile<DT, DC>;
    static constexpr int kTile = kRows * T::kRow, kBuffer = 2 * kTile, kLds = 2 * kBuffer;
};

template <int DT, int DC>
__global__ void __launch_bounds__(256, 1) attention_dkv_kernel(const Attention a) {
    using L = AttentionDkv<DT, DC>;
    using T = typename L::T;
    constexpr int SIZE = Operand<DT>::kSize, STEPS = DC / 16, DB = DC / 32;
    __shared__ __attribute__((aligned(16))) char lds_bytes[L::kLds];
    __shared__ __attribute__((aligned(16))) float lds_lse[2][L::kRows], lds_delta[2][L::kRows];
    __shared__ __attribute__((aligned(16))) int lds_seen[2][L::kRows];
    SDGP_SHARED char* lds = (SDGP_SHARED char*)lds_bytes;

    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const int head = blockIdx.x % a.Hk;
    Sequence s;
    int tile, tiles;
    if (!find_tile<true, L::kKeys>(a, blockIdx.x / a.Hk, s, tile, tiles)) return;   // the first keys have the most rows
    const int rows = s.nq * a.G, key0 = tile * L::kKeys + 32 * wave, key = key0 + (lane & 31);
    const auto seen = [&](int r) {
        return a.causal ? clamp_int((int)divide((uint32_t)r, a.by_group) + 1 + s.nk - s.nq, 0, s.nk) : s.nk;
    };
    const int width = key < s.nk ? a.D : 0;
    const int64_t key_row = s.k0 + (key < s.nk ? key : 0);
    Operand<DT> k[STEPS], v[STEPS];
    {
        const char* pk = static_cast<const char*>(a.k) + (key_row * a.k_token + (int64_t)head * a.k_head) * SIZE;
        const char* pv = static_cast<const char*>(a.v) + (key_row * a.v_token + (int64_t)head * a.v_head) * SIZE;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            k[i] = load_operand<DT>(pk, 16 * i + 8 * half, width);
            v[i] = load_operand<DT>(pv, 16 * i + 8 * half, width);
        }
    }
    // The first token that sees this tile's first key, and the tiles of rows from there on.
    int from = a.causal ? tile * L::kKeys + s.nq - s.nk : 0;
    from = clamp_int(from, 0, s.nq);
    const int begin = from * a.G / L::kRows, end = s.nk > 0 ? (rows + L::kRows - 1) / L::kRows : 0;

    Stage<DT, DC, L::kRows, L::kThreads> sq, sd;
    float next_lse = 0.0f, next_delta = 0.0f;
    int next_seen = 0;
    const auto fetch = [&](int n) {
        const auto place = [&](int r, int& tok, int& g) {
            const int at = n * L::kRows + r;
            tok = (int)divide((uint32_t)at, a.by_group), g = at - tok * a.G;
            return at < rows;
        };
        sq.load([&](int r) -> const char* {
            int tok, g;
            if (!place(r, tok, g)) return nullptr;
            return static_cast<const char*>(a.q) + ((int64_t)(s.q0 + tok) * a.q_token + (int64_t)(head * a.G + g) * a.q_head) * SIZE;
        }, a.D);
        sd.load([&](int r) -> const char* {
            int tok, g;
            if (!place(r, tok, g)) return nullptr;
            return static_cast<const char*>(a.d_o) + ((int64_t)(s.q0 + tok) * a.H + head * a.G + g) * a.D * SIZE;
        }, a.D);
        if ((int)threadIdx.x < L::kRows) {
            int tok, g;
            next_lse = next_delta = 0.0f, next_seen = 0x7FFFFFFF;        // rows behind the last: zeros throughout
            if (place((int)threadIdx.x, tok, g)) {
                const int64_t at = (int64_t)(s.q0 + tok) * a.H + head * a.G + g;
                next_lse = a.lse[at] * kLog2E, next_delta = a.delta[at];
                next_seen = seen(n * L::kRows + (int)threadIdx.x);
            }
        }
    };
    attn_f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dk[d][i] = dv[d][i] = 0.0f;
    if (begin < end) fetch(begin);
    for (int n = begin; n < end; ++n) {
        const int turn = n & 1;
        SDGP_SHARED char* qt = lds + turn * L::kBuffer;
        SDGP_SHARED char* dt = qt + L::kTile;
        sq.store(qt);
        sd.store(dt);
        if ((int)threadIdx.x < L::kRows)
            lds_lse[turn][threadIdx.x] = next_lse, lds_delta[turn][threadIdx.x] = next_delta, lds_seen[turn][threadIdx.x] = next_seen;
        __syncthreads();
        if (n + 1 < end) fetch(n + 1);
#pragma unroll
        for (int b = 0; b < L::kBlocks; ++b) {
            const int r0 = n * L::kRows + 32 * b, last = rows - 1 < r0 + 31 ? rows - 1 : r0 + 31;
            if (r0 >= rows || seen(last) <= key0) continue;
            attn_f32x16 x, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = dp[i] = 0.0f;
#pragma unroll
            for (int i = 0; i < STEPS; ++i) x = multiply(T::rows(qt, 32 * b, i, lane), k[i], x);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) dp = multiply(T::rows(dt, 32 * b, i, lane), v[i], dp);
            float p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = 32 * b + result_row(i, half);
                p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.c, -lds_lse[turn][r]));
            }
            if (seen(r0) < key0 + 32) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (key >= lds_seen[turn][32 * b + result_row(i, half)]) p[i] = 0.0f;
            }
            Operand<DT> po[2], ds[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float y[8], z[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int r = 32 * b + result_row(8 * u + i, half);
                    y[i] = p[8 * u + i];
                    z[i] = y[i] * (dp[8 * u + i] - lds_delta[turn][r]);
                }
                po[u].set(y);
                ds[u].set(z);
            }
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    dv[d] = multiply(T::columns(dt, 32 * b + 16 * u, d, lane), po[u], dv[d]);
                    dk[d] = multiply(T::columns(qt, 32 * b + 16 * u, d, lane), ds[u], dk[d]);
                }
        }
    }
    if (key >= s.nk) return;
    const int64_t to = (key_row * a.Hk + head) * a.D * SIZE;
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        store_block<DT>(static_cast<char*>(a.dk) + to, dk[d], d, half, a.D, a.scale);
        store_block<DT>(static_cast<char*>(a.dv) + to, dv[d], d, half, a.D, 1.0f);
    }
}

}  // namespace sdgp
