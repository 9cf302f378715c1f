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

template <int DT, int DC, bool FAST>
__global__ void __launch_bounds__(256, DT == SDGP_BF16 ? 2 : 1) attention_dq_kernel(const Attention a) {
    using L = AttentionDq<DT, DC>;
    using T = typename L::T;
    constexpr int SIZE = Operand<DT>::kSize, STEPS = DC / 16, DB = DC / 32;
    __shared__ __attribute__((aligned(512))) char lds_bytes[L::kLds];
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
            q[i] = load_operand<DT, FAST>(p, 16 * i + 8 * half, width);
            dO[i] = load_operand<DT, FAST>(pd, 16 * i + 8 * half, width);
            const Operand<DT> o = load_operand<DT, FAST>(po, 16 * i + 8 * half, width);
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

    Feed<DT, DC, L::kKeys, FAST> fk(keys, k_row, a.D), fv(values, v_row, a.D);
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
    attn_f32x16 dq[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dq[d][i] = 0.0f;
    if (end > 0) {
        start(0);
        finish(0);
    }
    for (int n = 0; n < end; ++n) {
        SDGP_SHARED char *kt = buffer(n), *vt = kt + L::kTile;
        if (n + 1 < end) start(n + 1);
        const uint32_t k_rows = T::rows_lane(kt, lane), v_rows = T::rows_lane(vt, lane), k_columns = T::columns_lane(kt, lane);
#pragma unroll
        for (int b = 0; b < L::kBlocks; ++b) {
            const int key0 = n * L::kKeys + 32 * b;
            if (key0 >= most_mine || !any_row) continue;
            attn_f32x16 x, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = dp[i] = 0.0f;
#pragma unroll
            for (int i = 0; i < STEPS; ++i) x = multiply(T::rows(k_rows, 32 * b, i), q[i], x);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) dp = multiply(T::rows(v_rows, 32 * b, i), dO[i], dp);
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
                for (int u = 0; u < 2; ++u) dq[d] = multiply(T::columns(k_columns, 32 * b + 16 * u, d), ds[u], dq[d]);
        }
        if (n + 1 < end) finish(n + 1);
    }
    if (row >= rows) return;
#pragma unroll
    for (int d = 0; d < DB; ++d) store_block<DT>(static_cast<char*>(a.dq) + out_row * a.D * SIZE, dq[d], d, half, a.D, a.scale);
}

// The queries pass by in tiles of kRows tokens of one head; a group's heads one after the other.
template <int DT, int DC>
struct AttentionDkv {
    static constexpr int kThreads = 256, kKeys = 128, kRows = DT == SDGP_BF16 ? 64 : 32, kBlocks = kRows / 32;
    using T = Tile<DT, DC>;
    static constexpr int kTile = kRows * T::kRow, kBuffer = 2 * kTile, kLds = 2 * kBuffer;
};

template <int DT, int DC, bool FAST>
__global__ void __launch_bounds__(256, DT == SDGP_BF16 ? 2 : 1) attention_dkv_kernel(const Attention a) {
    using L = AttentionDkv<DT, DC>;
    using T = typename L::T;
    constexpr int SIZE = Operand<DT>::kSize, STEPS = DC / 16, DB = DC / 32, NB = L::kBlocks;
    __shared__ __attribute__((aligned(512))) char lds_bytes[L::kLds];
    __shared__ __attribute__((aligned(16))) float lds_lse[2][L::kRows], lds_delta[2][L::kRows];
    SDGP_SHARED char* lds = (SDGP_SHARED char*)lds_bytes;

    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const int head = blockIdx.x % a.Hk;
    Sequence s;
    int tile, tiles;
    if (!find_tile<true, L::kKeys>(a, blockIdx.x / a.Hk, s, tile, tiles)) return;   // the first keys have the most rows
    const int key0 = tile * L::kKeys + 32 * wave, key = key0 + (lane & 31);
    const int ahead = s.nk - s.nq;                                      // token t sees the keys up to t + ahead, if causal
    const int width = key < s.nk ? a.D : 0;
    const int64_t key_row = s.k0 + (key < s.nk ? key : 0);
    Operand<DT> k[STEPS], v[STEPS];
    {
        const char* pk = static_cast<const char*>(a.k) + (key_row * a.k_token + (int64_t)head * a.k_head) * SIZE;
        const char* pv = static_cast<const char*>(a.v) + (key_row * a.v_token + (int64_t)head * a.v_head) * SIZE;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            k[i] = load_operand<DT, FAST>(pk, 16 * i + 8 * half, width);
            v[i] = load_operand<DT, FAST>(pv, 16 * i + 8 * half, width);
        }
    }
    // The first token that sees this tile's first key, and the tiles of tokens from there on, of each head.
    const int from = a.causal ? clamp_int(tile * L::kKeys - ahead, 0, s.nq) : 0;
    const int first = from / L::kRows, each = s.nk > 0 ? (s.nq + L::kRows - 1) / L::kRows - first : 0, end = each * a.G;

    const int64_t q_row = a.q_token * SIZE, d_row = (int64_t)a.H * a.D * SIZE;
    const char* queries = static_cast<const char*>(a.q) + ((int64_t)s.q0 * a.q_token + (int64_t)head * a.G * a.q_head) * SIZE;
    const char* grads = static_cast<const char*>(a.d_o) + ((int64_t)s.q0 * a.H + head * a.G) * a.D * SIZE;
    Feed<DT, DC, L::kRows, FAST> fq(queries, q_row, a.D), fd(grads, d_row, a.D);
    float next_lse = 0.0f, next_delta = 0.0f;
    int next = first, g = 0;                                            // the tile that is asked for next, and its head
    const auto buffer = [&](int n) { return lds + (n & 1) * L::kBuffer; };
    const auto start = [&](int n) {
        fq.start(buffer(n), next * L::kRows, s.nq);
        fd.start(buffer(n) + L::kTile, next * L::kRows, s.nq);
        if ((int)threadIdx.x < L::kRows) {
            const int t = next * L::kRows + (int)threadIdx.x;
            next_lse = next_delta = 0.0f;                               // tokens behind the last: zeros throughout
            if (t < s.nq) {
                const int64_t at = (int64_t)(s.q0 + t) * a.H + head * a.G + g;
                next_lse = a.lse[at] * kLog2E, next_delta = a.delta[at];
            }
        }
        if (++next == first + each) {
            next = first, ++g;
            fq.base += a.q_head * SIZE;
            fd.base += a.D * SIZE;
        }
    };
    const auto finish = [&](int n) {
        fq.finish(buffer(n));
        fd.finish(buffer(n) + L::kTile);
        if ((int)threadIdx.x < L::kRows) lds_lse[n & 1][threadIdx.x] = next_lse, lds_delta[n & 1][threadIdx.x] = next_delta;
        __syncthreads();
    };
    attn_f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) dk[d][i] = dv[d][i] = 0.0f;
    // One block of 32 tokens.  Operands from LDS are asked for kAhead products before they are needed, and no earlier: the keys'
    // operands and sums fill three quarters of the registers of two wavefronts a SIMD, which cover each other's other work.
    const auto block = [&](int b, int turn, int t0, bool masked) __attribute__((always_inline)) {
        constexpr int kAhead = 2;
        SDGP_SHARED char* tiles = lds + turn * L::kBuffer + b * 32 * T::kRow;    // of queries, and kTile on of gradients
        Operand<DT> f[kAhead + 1];
        attn_f32x16 x, dp;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = dp[i] = 0.0f;
        const uint32_t rows_at = here(T::rows_lane(tiles, lane));
        const auto rows = [&](int i) { return i < STEPS ? T::rows(rows_at, 0, i) : T::rows(rows_at, 0, i - STEPS, L::kTile); };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) f[i] = rows(i);
#pragma unroll
        for (int i = 0; i < 2 * STEPS; ++i) {
            if (i + kAhead < 2 * STEPS) f[(i + kAhead) % (kAhead + 1)] = rows(i + kAhead);
            __builtin_amdgcn_sched_barrier(0);
            if (i < STEPS) x = multiply(f[i % (kAhead + 1)], k[i], x);
            else dp = multiply(f[i % (kAhead + 1)], v[i - STEPS], dp);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = 32 * b + result_row(i, half);
            x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.c, -lds_lse[turn][r]));
            dp[i] = x[i] * (dp[i] - lds_delta[turn][r]);
        }
        if (masked) {
            const int behind = (int)here((uint32_t)(key - t0 - ahead - 4 * half));   // (and not without the branch)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (behind > result_row(i, 0)) x[i] = dp[i] = 0.0f;
        }
        Operand<DT> p[2], ds[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float y[8], z[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = x[8 * u + i], z[i] = dp[8 * u + i];
            p[u].set(y);
            ds[u].set(z);
        }
        __builtin_amdgcn_sched_barrier(0);
        // dv and dk in turn: block i / 4, rows 16 (i / 2 % 2) ..
        const uint32_t columns_at = here(T::columns_lane(tiles, lane));
        const auto columns = [&](int i) { return T::columns(columns_at, 16 * (i / 2 & 1), i / 4, i & 1 ? 0 : L::kTile); };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) f[i] = columns(i);
#pragma unroll
        for (int i = 0; i < 4 * DB; ++i) {
            if (i + kAhead < 4 * DB) f[(i + kAhead) % (kAhead + 1)] = columns(i + kAhead);
            __builtin_amdgcn_sched_barrier(0);
            if (i & 1) dk[i / 4] = multiply(f[i % (kAhead + 1)], ds[i / 2 & 1], dk[i / 4]);
            else dv[i / 4] = multiply(f[i % (kAhead + 1)], p[i / 2 & 1], dv[i / 4]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (end > 0) {
        start(0);
        finish(0);
    }
    int now = first;
    for (int n = 0; n < end; ++n) {
        if (n + 1 < end) start(n + 1);
        const int turn = n & 1, t0 = now * L::kRows;
        if (++now == first + each) now = first;
        if (key0 < s.nk) {
#pragma unroll 1
            for (int b = 0; b < NB; ++b) {
                const int at = t0 + 32 * b;
                if (a.causal && at + 31 + ahead < key0) continue;       // none of the tokens sees any of the keys
                block(b, turn, at, a.causal && at + ahead < key0 + 31);
            }
        }
        if (n + 1 < end) finish(n + 1);
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
