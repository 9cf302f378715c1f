// Gradients of attention, from dO, the inputs, o and lse.
//
//   P = exp(scale q k^T - lse),  delta = sum_d dO o = sum over keys of P dP,  dP = dO V^T,  dS = P (dP - delta)
//   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO, the latter two summed over a key head's queries
// Two kernels without atomics: one owns queries and passes over the keys (dQ, and delta on the way), one owns keys and passes
// over the queries (dK, dV).  Each computes the scores again: 7 products of 2 D flops a pair instead of 5, for sums in
// a fixed order that are read and written once.  As forward, every 32x32 result stands in the registers as the next
// product's operand: with the owned rows in the results' columns, a lane holds sixteen of the passing rows.  P and dS are rounded
// to bf16 for bf16 tensors, as operands of bf16 products; the sums are fp32.  delta: dO o carries o's own rounding, which the other
// sum does not; it is there once the keys have passed, so it is the keys' kernel's, and dQ's too where one tile holds all of a
// workgroup's keys (64 sequences of 32 tokens: dQ and dK off by 0.0024 of their size against 64 bits, 0.0030 with dO o).
#pragma once

#include "attention.h"

namespace sdgp {

constexpr float kLog2E = 1.44269504088896341f;

// Four wavefronts, OWN of them with 32 owned rows (or keys) each; the others share those and take every second block of what
// passes by, their sums being added at the end: twice the workgroups, for problems of few.
template <int DT, int DC, int OWN>
struct AttentionDq {
    static constexpr int kRows = 32 * OWN, kShare = 4 / OWN, kKeys = DT == SDGP_BF16 || kShare > 1 ? 64 : 32, kBlocks = kKeys / 32;
    using T = Tile<DT, DC>;
    static constexpr int kTile = kKeys * T::kRow, kBuffer = 2 * kTile, kLds = 2 * kBuffer;
};

// Adds the sums of wavefronts OWN .. 3 to those of the ones that own the same rows.  All threads call it, and LDS is free.
template <int OWN, int N>
__device__ __forceinline__ void add_shared(SDGP_SHARED char* lds, int wave, int lane, attn_f32x16 (&x)[N]) {
    if constexpr (OWN == 4) return;
    SDGP_SHARED float* sums = (SDGP_SHARED float*)lds;                  // [OWN, N, 16, 64]
    __syncthreads();
    if (wave >= OWN) {
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) sums[(((wave - OWN) * N + d) * 16 + i) * 64 + lane] = x[d][i];
    }
    __syncthreads();
    if (wave < OWN) {
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[d][i] += sums[((wave * N + d) * 16 + i) * 64 + lane];
    }
}

template <int DT, int DC, bool FAST, int OWN>
__global__ void __launch_bounds__(256, DT == SDGP_BF16 ? 2 : 1) attention_dq_kernel(const Attention a) {
    using L = AttentionDq<DT, DC, OWN>;
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
    const int own = wave % OWN, first_row = row0 + 32 * own, row = first_row + (lane & 31);
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
    if (row < rows && half == 0 && wave == own) a.lse2[out_row] = lse2;

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
    float passed = 0.0f;                                                // sum of P dP
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
        for (int pass = end == 1 ? 0 : 1; pass < 2; ++pass) {
            const bool last_pass = pass == 1;
#pragma unroll
            for (int b = 0; b < L::kBlocks; ++b) {
                const int key0 = n * L::kKeys + 32 * b;
                if (key0 >= most_mine || !any_row || (L::kShare > 1 && last_pass && (b & 1) != wave / OWN)) continue;
                attn_f32x16 x, dp;
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = dp[i] = 0.0f;
#pragma unroll
                for (int i = 0; i < STEPS; ++i) x = multiply(T::rows(k_rows, 32 * b, i), q[i], x);
#pragma unroll
                for (int i = 0; i < STEPS; ++i) dp = multiply(T::rows(v_rows, 32 * b, i), dO[i], dp);
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.c, -lse2));
                if (key0 + 32 > fewest) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (key0 + result_row(i, half) >= mine) x[i] = 0.0f;
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) passed = __builtin_fmaf(x[i], dp[i], passed);
                if (!last_pass) continue;
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] *= dp[i] - delta;
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
            if (!last_pass) delta = halves_sum(passed), passed = 0.0f;  // (of all the keys: no wavefront has left any out)
        }
        if (n + 1 < end) finish(n + 1);
    }
    add_shared<OWN>(lds, wave, lane, dq);
    passed = halves_sum(passed);
    if constexpr (L::kShare > 1) {
        __shared__ float lds_passed[32 * OWN];
        if (wave >= OWN && half == 0) lds_passed[32 * own + lane] = passed;
        __syncthreads();
        if (wave < OWN) passed += lds_passed[32 * own + (lane & 31)];
    }
    if (row >= rows || wave != own) return;
    if (half == 0) a.delta[out_row] = passed;
#pragma unroll
    for (int d = 0; d < DB; ++d) store_block<DT, FAST>(static_cast<char*>(a.dq) + out_row * a.D * SIZE, dq[d], d, half, a.D, a.scale);
}

// The queries pass by in tiles of some tokens of all the group's heads, the sequence's last tokens first: so workgroups that started
// together read the same tiles at the same time, whichever their keys are.  (Tiles of one head: 1255 us instead of 820 for 22294 packed
// tokens of 16 heads.  Their rows are 4096 bytes apart in dO, where memory's channels repeat.)
template <int DT, int DC, int OWN>
struct AttentionDkv {
    // Of bf16 heads of 128, the sums fill half the registers of two wavefronts a SIMD and the keys' operands an eighth; the values'
    // come from LDS, since what does not fit is kept in memory, whose loads wait for the tiles on their way.
    static constexpr bool kValuesInLds = DT == SDGP_BF16 && DC > 96;
    static constexpr int kKeys = 32 * OWN, kShare = 4 / OWN, kRows = attention_dkv_rows(DT, DC, OWN), kBlocks = kRows / 32;
    using T = Tile<DT, DC>;
    static constexpr int kTile = kRows * T::kRow, kBuffer = 2 * kTile, kValues = 2 * kBuffer, kLds = kValues + (kValuesInLds ? kKeys * T::kRow : 0);
};

template <int DT, int DC, bool FAST, int OWN>
__global__ void __launch_bounds__(256, DT == SDGP_BF16 ? 2 : 1) attention_dkv_kernel(const Attention a) {
    using L = AttentionDkv<DT, DC, OWN>;
    using T = typename L::T;
    constexpr int SIZE = Operand<DT>::kSize, STEPS = DC / 16, DB = DC / 32, NB = L::kBlocks;
    __shared__ __attribute__((aligned(512))) char lds_bytes[L::kLds];
    __shared__ __attribute__((aligned(16))) float lds_rows[2][2][64];     // lse2 and delta of a tile's rows
    __shared__ __attribute__((aligned(16))) int lds_token[L::kRows];      // a row's token in its tile
    SDGP_SHARED char* lds = (SDGP_SHARED char*)lds_bytes;

    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const int head = blockIdx.x % a.Hk, rest = blockIdx.x / a.Hk, part = rest % a.parts;
    Sequence s;
    int tile, tiles;
    if (!find_tile<true, L::kKeys>(a, rest / a.parts, s, tile, tiles)) return;      // the first keys have the most rows
    const int own = wave % OWN, key0 = tile * L::kKeys + 32 * own, key = key0 + (lane & 31);
    const int ahead = s.nk - s.nq;                                      // token t sees the keys up to t + ahead, if causal
    const int width = key < s.nk ? a.D : 0;
    const int64_t key_row = s.k0 + (key < s.nk ? key : 0);
    Operand<DT> k[STEPS], v[L::kValuesInLds ? 1 : STEPS];
    {
        const char* pk = static_cast<const char*>(a.k) + (key_row * a.k_token + (int64_t)head * a.k_head) * SIZE;
        const char* pv = static_cast<const char*>(a.v) + (key_row * a.v_token + (int64_t)head * a.v_head) * SIZE;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            k[i] = load_operand<DT, FAST>(pk, 16 * i + 8 * half, width);
            const Operand<DT> x = load_operand<DT, FAST>(pv, 16 * i + 8 * half, width);
            if constexpr (L::kValuesInLds) {
                if (wave == own) *(SDGP_SHARED attn_u32x4*)(lds + L::kValues + T::at(32 * own + (lane & 31), 2 * i + half)) = __builtin_bit_cast(attn_u32x4, x);
            } else {
                v[i] = x;
            }
        }
    }
    // A tile's tokens and heads, the first token that sees this tile's first key, and the tiles of tokens from there on.
    const int heads = a.G < L::kRows ? a.G : L::kRows, tokens = L::kRows / heads, chunks = (a.G + heads - 1) / heads;
    const int from = a.causal ? clamp_int(tile * L::kKeys - ahead, 0, s.nq) : 0;
    const int first = from / tokens, each = s.nk > 0 ? (s.nq + tokens - 1) / tokens - first : 0, all = (each > 0 ? each : 0) * chunks;
    const int per = (all + a.parts - 1) / a.parts, begin = part * per < all ? part * per : all, end = begin + per < all ? begin + per : all;

    const char* queries = static_cast<const char*>(a.q) + ((int64_t)s.q0 * a.q_token + (int64_t)head * a.G * a.q_head) * SIZE;
    const char* grads = static_cast<const char*>(a.d_o) + ((int64_t)s.q0 * a.H + head * a.G) * a.D * SIZE;
    FeedQueries<DT, DC, L::kRows, FAST> fq(queries, a.q_token * SIZE, a.q_head * SIZE, a.D), fd(grads, (int64_t)a.H * a.D * SIZE, (int64_t)a.D * SIZE, a.D);
    int chunk = begin % chunks, next = first + each - 1 - begin / chunks;   // the heads and tile that are asked for next
    int now_chunk = chunk, now = next;                                  // .. that are worked on
    if ((int)threadIdx.x < L::kRows) lds_token[threadIdx.x] = (int)divide(threadIdx.x, a.by_heads);
    const auto buffer = [&](int n) { return lds + (n & 1) * L::kBuffer; };
    const auto start = [&](int n) {
        const int t0 = next * tokens, g0 = chunk * heads, has = s.nq - t0, wide = a.G - g0 < heads ? a.G - g0 : heads;
        const int lasting = has < tokens ? has : tokens;
        fq.base = queries + (t0 * fq.row + g0 * fq.head);
        fd.base = grads + (t0 * fd.row + g0 * fd.head);
        fq.start(buffer(n), a.by_heads, heads, lasting, wide);
        fd.start(buffer(n) + L::kTile, a.by_heads, heads, lasting, wide);
        if (wave < 2) {                                                 // (one wavefront each; rows that are not there: zeros throughout)
            const int t = (int)divide((uint32_t)lane, a.by_heads), g = lane - t * heads;
            const float* of = (wave == 0 ? a.lse2 : a.delta) + ((int64_t)(s.q0 + t0) * a.H + head * a.G + g0);
            copy_to_lds<4>(records(of, kNoRecord), lane < L::kRows && t < lasting && g < wide ? (uint32_t)(t * a.H + g) * 4u : kNoRecord,
                           (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(SDGP_SHARED float*)lds_rows[n & 1][wave]));
        }
        if (++chunk == chunks) chunk = 0, --next;
    };
    const auto finish = [&](int n) {
        fq.finish(buffer(n));
        fd.finish(buffer(n) + L::kTile);
        wait_for_copies();
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
        constexpr int kAhead = L::kValuesInLds ? 2 : 3, kAheadOut = 4;
        SDGP_SHARED char* tiles = lds + turn * L::kBuffer + b * 32 * T::kRow;    // of queries, and kTile on of gradients
        Operand<DT> f[kAhead + 1];
        attn_f32x16 x, dp;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = dp[i] = 0.0f;
        const uint32_t rows_at = here(T::rows_lane(tiles, lane));
        Operand<DT> fv[kAhead + 1];
        const uint32_t values_at = L::kValuesInLds ? here(T::rows_lane(lds + L::kValues + own * 32 * T::kRow, lane)) : 0;
        const auto rows = [&](int i) { return i < STEPS ? T::rows(rows_at, 0, i) : T::rows(rows_at, 0, i - STEPS, L::kTile); };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) f[i] = rows(i);
#pragma unroll
        for (int i = 0; i < 2 * STEPS; ++i) {
            if (i + kAhead < 2 * STEPS) f[(i + kAhead) % (kAhead + 1)] = rows(i + kAhead);
            if (L::kValuesInLds && i + kAhead >= STEPS && i + kAhead < 2 * STEPS)
                fv[(i + kAhead - STEPS) % (kAhead + 1)] = T::rows(values_at, 0, i + kAhead - STEPS);
            __builtin_amdgcn_sched_barrier(0);
            if (i < STEPS) x = multiply(f[i % (kAhead + 1)], k[i], x);
            else if constexpr (L::kValuesInLds) dp = multiply(f[i % (kAhead + 1)], fv[(i - STEPS) % (kAhead + 1)], dp);
            else dp = multiply(f[i % (kAhead + 1)], v[i - STEPS], dp);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = 32 * b + result_row(i, half);
            x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.c, -lds_rows[turn][0][r]));
            dp[i] = x[i] * (dp[i] - lds_rows[turn][1][r]);
        }
        if (masked) {
            const int mine = (int)here((uint32_t)(key - t0 - ahead));   // (and not without the branch)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (mine > lds_token[32 * b + result_row(i, half)]) x[i] = dp[i] = 0.0f;
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
        Operand<DT> h[kAheadOut + 1];
        const uint32_t columns_at = here(T::columns_lane(tiles, lane));
        const auto columns = [&](int i) { return T::columns(columns_at, 16 * (i / 2 & 1), i / 4, i & 1 ? 0 : L::kTile); };
#pragma unroll
        for (int i = 0; i < kAheadOut; ++i) h[i] = columns(i);
#pragma unroll
        for (int i = 0; i < 4 * DB; ++i) {
            if (i + kAheadOut < 4 * DB) h[(i + kAheadOut) % (kAheadOut + 1)] = columns(i + kAheadOut);
            __builtin_amdgcn_sched_barrier(0);
            if (i & 1) dk[i / 4] = multiply(h[i % (kAheadOut + 1)], ds[i / 2 & 1], dk[i / 4]);
            else dv[i / 4] = multiply(h[i % (kAheadOut + 1)], p[i / 2 & 1], dv[i / 4]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (begin < end) {
        start(begin);
        finish(begin);
    }
    for (int n = begin; n < end; ++n) {
        if (n + 1 < end) start(n + 1);
        const int turn = n & 1, t0 = now * tokens;
        if (++now_chunk == chunks) now_chunk = 0, --now;
        if (key0 < s.nk) {
#pragma unroll 1
            for (int b = 0; b < NB; ++b) {
                if (L::kShare > 1 && (b & 1) != wave / OWN) continue;   // another wavefront's
                // the last key that the block's first and last rows see
                const int low = t0 + (int)divide((uint32_t)(32 * b), a.by_heads) + ahead, high = t0 + (int)divide((uint32_t)(32 * b + 31), a.by_heads) + ahead;
                if (a.causal && high < key0) continue;
                block(b, turn, t0, a.causal && low < key0 + 31);
            }
        }
        if (n + 1 < end) finish(n + 1);
    }
    add_shared<OWN>(lds, wave, lane, dk);
    add_shared<OWN>(lds, wave, lane, dv);
    if (key >= s.nk || wave != own) return;
    const int64_t to = (key_row * a.Hk + head) * a.D;
    if (a.parts > 1) {
        float* pk = a.part_o + (int64_t)part * 2 * a.Tk * a.Hk * a.D + to;
        float* pv = pk + (int64_t)a.Tk * a.Hk * a.D;
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            store_block<SDGP_F32, FAST>(reinterpret_cast<char*>(pk), dk[d], d, half, a.D, a.scale);
            store_block<SDGP_F32, FAST>(reinterpret_cast<char*>(pv), dv[d], d, half, a.D, 1.0f);
        }
        return;
    }
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        store_block<DT, FAST>(static_cast<char*>(a.dk) + to * SIZE, dk[d], d, half, a.D, a.scale);
        store_block<DT, FAST>(static_cast<char*>(a.dv) + to * SIZE, dv[d], d, half, a.D, 1.0f);
    }
}

// dk and dv from the parts' sums [parts, 2, Tk Hk D], four values a thread (fewer at the end of each).
template <int DT>
__global__ void __launch_bounds__(256) attention_dkv_join(const Attention a) {
    typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4), may_alias));
    const int64_t n = (int64_t)a.Tk * a.Hk * a.D, fours = (n + 3) / 4;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < 2 * fours; e += (int64_t)gridDim.x * 256) {
        const int64_t at = (e < fours ? e : e - fours) * 4;
        const float* from = a.part_o + (e < fours ? 0 : n) + at;
        const int left = (int)(n - at < 4 ? n - at : 4);
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (left == 4) {
#pragma unroll 4
            for (int p = 0; p < a.parts; ++p) {
                const f32x4 x = *reinterpret_cast<const f32x4*>(from + (int64_t)p * 2 * n);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] += x[i];
            }
        } else {
            for (int p = 0; p < a.parts; ++p)
                for (int i = 0; i < 3; ++i)
                    if (i < left) sum[i] += from[(int64_t)p * 2 * n + i];
        }
        void* to = e < fours ? a.dk : a.dv;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i >= left) break;
            if constexpr (DT == SDGP_BF16) static_cast<uint16_t*>(to)[at + i] = (uint16_t)float_to_bf16(sum[i]);
            else static_cast<float*>(to)[at + i] = sum[i];
        }
    }
}

}  // namespace sdgp
