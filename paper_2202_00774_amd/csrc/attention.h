// Attention over packed sequences: arguments, where a workgroup's tile lies, and tiles in LDS as the matrix instructions
// take them.  The kernels' mathematics stands in attention_fwd.h and attention_bwd.h.
#pragma once

#include <type_traits>

#include "common.h"
#include "fastdiv.h"

namespace sdgp {

#define SDGP_SHARED __attribute__((address_space(3)))

struct Attention {
    const void *q, *k, *v;
    int64_t q_token, q_head, k_token, k_head, v_token, v_head;   // strides in elements
    const int32_t *off_q, *off_k, *len_k;                        // null: S sequences of Lq and Lk tokens each
    int S, Lq, Lk, Tq, Tk, H, Hk, G, D, causal, buckets;
    FastDiv by_group, by_heads;                                  // rows / G; a tile's rows / its heads (backward)
    float scale, c;                                              // c = scale log2 e
    bool fast;                                                   // Feed<..., FAST>
    void* o;
    float* lse;
    int parts;                                                   // pieces of a row's keys (forward), of a key's rows (backward)
    float *part_o, *part_ml;                                     // forward: [parts, Tq H, D], [parts, Tq H, 2]; backward: [parts, 2, Tk Hk, D]
    const void *d_o, *o_in;
    float *lse2, *delta;                                         // [Tq H]: lse log2 e, and sum of dO o
    void *dq, *dk, *dv;
};

// Wavefronts of the keys' gradients' workgroups with keys of their own (fp32: two, whose tiles fill LDS already).
constexpr int attention_own_keys(int dt) { return dt == SDGP_BF16 ? 4 : 2; }

// How the gradients' kernels cut the work: wavefronts of a workgroup with rows of their own, tiles of each.
struct AttentionGrid {
    int own_rows;
    int64_t row_tiles, key_tiles;
};

// Rows of queries in a tile of the keys' gradients' kernel, as LDS holds them; DC: values of a head as the kernel counts them.
constexpr int attention_dkv_rows(int dt, int DC, int own) { return own < 4 || (dt == SDGP_BF16 && DC <= 96) ? 64 : 32; }

// A key head's queries are the rows (token, head of the group), token by token: its keys are read once for all heads of
// the group, and their gradients are sums over these rows.
struct Sequence {
    int q0, nq, k0, nk;
};

__device__ __forceinline__ int clamp_int(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

// The tokens of sequence i; offsets that are wrong stay within the tensors.
__device__ __forceinline__ Sequence sequence_at(const Attention& a, int i) {
    Sequence s;
    if (a.off_q) {
        s.q0 = clamp_int(a.off_q[i], 0, a.Tq);
        s.nq = clamp_int(a.off_q[i + 1], s.q0, a.Tq) - s.q0;
        s.k0 = clamp_int(a.off_k[i], 0, a.Tk);
        s.nk = clamp_int(a.off_k[i + 1], s.k0, a.Tk) - s.k0;
    } else {
        s.q0 = i * a.Lq, s.nq = a.Lq;
        s.k0 = i * a.Lk, s.nk = a.len_k ? clamp_int(a.len_k[i], 0, a.Lk) : a.Lk;
    }
    return s;
}

// Rows that no sequence holds: in front of the first one (i == -1) and behind the last (i == S).  They see nothing.
template <bool KEYS>
__device__ __forceinline__ Sequence rows_outside(const Attention& a, bool behind) {
    const int T = KEYS ? a.Tk : a.Tq;
    const int32_t* off = KEYS ? a.off_k : a.off_q;
    const int at = clamp_int(off[behind ? a.S : 0], 0, T);
    Sequence s = {0, 0, 0, 0};
    if (KEYS) s.k0 = behind ? at : 0, s.nk = behind ? T - at : at;
    else s.q0 = behind ? at : 0, s.nq = behind ? T - at : at;
    return s;
}

// How many of a sequence's tiles of UNIT rows (KEYS: of keys; else of queries, G a token) have at least `work` to do: of keys,
// the tokens that see the first one; of queries, the keys that the last one sees.
template <bool KEYS, int UNIT>
__device__ __forceinline__ int tiles_of_work(const Attention& a, const Sequence& s, int work) {
    const int tiles = ((KEYS ? s.nk : s.nq * a.G) + UNIT - 1) / UNIT;
    if (work <= 0) return tiles;
    if (work > (KEYS ? s.nq : s.nk)) return 0;
    if (!a.causal) return tiles;
    if (KEYS) return s.nk < work ? 0 : clamp_int((s.nk - work) / UNIT + 1, 0, tiles);
    const int token = work - 1 - s.nk + s.nq;                           // the first one that sees so many
    return token <= 0 ? tiles : token >= s.nq ? 0 : tiles - token * a.G / UNIT;
}

// Workgroup `index`'s tile of UNIT rows: false if it has none.  `tile` counts a sequence's tiles from the one with the most work.
//
// With offsets, each sequence has the tiles from (rows in front of it) / UNIT + its number on, which leaves it room for the one that
// is not full: a wavefront looks at 64 places at once (every wavefront for itself; the results are uniform; adding up the sequences'
// tiles instead took 250 us a call, waited for, on 4096 sequences of one token, 2500 on 16384, and this 85 and 200).  With a.buckets, of up to
// kInOrder sequences, a lane has one of them, and those tiles come first that have three quarters of the most work there is, then those
// with half of it, and so on: the long ones start first, and workgroups that run together share their sequences' rows as far as they can.
constexpr int kInOrder = 62;                                     // and the rows in front of the first and behind the last

template <bool KEYS, int UNIT>
__device__ __forceinline__ bool find_tile(const Attention& a, int index, Sequence& s, int& tile, int& tiles) {
    if (a.off_q == nullptr) {
        tiles = ((KEYS ? a.Lk : a.Lq * a.G) + UNIT - 1) / UNIT;
        const int i = index / tiles;
        if (i >= a.S) return false;
        s = sequence_at(a, i);
        if (KEYS) s.nk = a.Lk;                                   // (lengths: forward only)
        tile = index - i * tiles;
        return true;
    }
    const int lane = threadIdx.x & 63;
    const auto sequence = [&](int i) {
        Sequence x = {0, 0, 0, 0};
        if (i <= a.S) x = i >= 0 && i < a.S ? sequence_at(a, i) : rows_outside<KEYS>(a, i >= 0);
        return x;
    };
    if (a.buckets == 1) {
        const int T = KEYS ? a.Tk : a.Tq;
        const int32_t* off = KEYS ? a.off_k : a.off_q;
        const auto place = [&](int i) { return (i == 0 ? 0 : clamp_int(off[i - 1], 0, T)) * (KEYS ? 1 : a.G) / UNIT + i; };
        int low = 0, high = a.S + 2;                             // the last of these whose place is not behind index
        while (high - low > 1) {
            const int step = (high - low + 63) / 64, at = low + lane * step;
            const uint64_t there = __ballot(at < high && place(at < high ? at : low) <= index);
            low += there == 0 ? 0 : (63 - __builtin_clzll(there)) * step;
            high = low + step < high ? low + step : high;
        }
        s = sequence(low - 1);                                   // (one for all lanes, which the compiler does not see)
        s.q0 = __builtin_amdgcn_readfirstlane(s.q0), s.nq = __builtin_amdgcn_readfirstlane(s.nq);
        s.k0 = __builtin_amdgcn_readfirstlane(s.k0), s.nk = __builtin_amdgcn_readfirstlane(s.nk);
        low = __builtin_amdgcn_readfirstlane(low);
        tiles = ((KEYS ? s.nk : s.nq * a.G) + UNIT - 1) / UNIT;
        tile = index - place(low);
        return tile >= 0 && tile < tiles;
    }
    const Sequence mine = sequence(lane - 1);
    int most = KEYS ? mine.nq : mine.nk;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_xor(most, o);
        most = most < x ? x : most;
    }
    int before = 0;
    for (int b = a.buckets - 1; b >= 0; --b) {
        const int low = (int)((int64_t)most * b / a.buckets), high = b == a.buckets - 1 ? 0x7FFFFFFF : (int)((int64_t)most * (b + 1) / a.buckets);
        const int above = tiles_of_work<KEYS, UNIT>(a, mine, high), n = tiles_of_work<KEYS, UNIT>(a, mine, b == 0 ? 0 : low) - above;
        int upto = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(upto, o);
            if (lane >= o) upto += x;
        }
        const uint64_t past = __ballot(before + upto > index);
        if (past != 0) {
            const int at = __builtin_ctzll(past);
            s.q0 = __builtin_amdgcn_readlane(mine.q0, at), s.nq = __builtin_amdgcn_readlane(mine.nq, at);
            s.k0 = __builtin_amdgcn_readlane(mine.k0, at), s.nk = __builtin_amdgcn_readlane(mine.nk, at);
            tiles = ((KEYS ? s.nk : s.nq * a.G) + UNIT - 1) / UNIT;
            tile = index - before - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(n, at)) + __builtin_amdgcn_readlane(above, at);
            return true;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// Workgroups that have all of find_tile's tiles.
inline int64_t most_tiles(bool packed, int64_t S, int64_t T, int64_t L, int64_t each, int64_t unit) {
    return packed ? T * each / unit + S + 2 : S * ((L * each + unit - 1) / unit);
}

// ------------------------------------------------------------------------------------------- operands and tiles

typedef __bf16 attn_bf16x8 __attribute__((ext_vector_type(8)));
typedef short attn_s16x4 __attribute__((ext_vector_type(4)));
typedef short attn_s16x8 __attribute__((ext_vector_type(8)));
typedef float attn_f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t attn_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t attn_u32x4_half __attribute__((ext_vector_type(4), aligned(2), may_alias));

// Eight values of the summed axis for a lane's row: lanes 0 .. 31 hold rows 0 .. 31 and the first eight of sixteen steps,
// lanes 32 .. 63 the same rows and the other eight.  fp32 values are multiplied one a half at a time (32x32x2); which eight
// belong together is the same for both operands, so their order is free.
template <int DT>
struct Operand;

template <>
struct Operand<SDGP_BF16> {
    static constexpr int kSize = 2;
    attn_u32x4 w;
    __device__ __forceinline__ void set(const float (&x)[8]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = float2_to_bf16x2(x[2 * i], x[2 * i + 1]);
    }
    __device__ __forceinline__ float get(int i) const { return bits_to_float((i & 1) ? (w[i / 2] & 0xFFFF0000u) : (w[i / 2] << 16)); }
};

template <>
struct Operand<SDGP_F32> {
    static constexpr int kSize = 4;
    float x[8];
    __device__ __forceinline__ void set(const float (&y)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = y[i];
    }
    __device__ __forceinline__ float get(int i) const { return x[i]; }
};

__device__ __forceinline__ attn_f32x16 multiply(const Operand<SDGP_BF16>& a, const Operand<SDGP_BF16>& b, attn_f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(attn_bf16x8, a.w), __builtin_bit_cast(attn_bf16x8, b.w), c, 0, 0, 0);
}
__device__ __forceinline__ attn_f32x16 multiply(const Operand<SDGP_F32>& a, const Operand<SDGP_F32>& b, attn_f32x16 c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x[i], b.x[i], c, 0, 0, 0);
    return c;
}

// Row of element i (of 16) of a 32x32 result; the column is lane % 32.
__device__ __forceinline__ int result_row(int i, int half) { return 8 * (i / 4) + 4 * half + i % 4; }

// Sixteen bytes of a row of n elements from element e on; what lies outside is 0 and is not read.  Rows begin anywhere.
template <int DT>
__device__ __forceinline__ attn_u32x4 load_chunk(const char* row, int e, int n) {
    constexpr int N = 16 / Operand<DT>::kSize;
    if (e + N <= n) return *reinterpret_cast<const attn_u32x4_half*>(row + e * Operand<DT>::kSize);
    union {
        attn_u32x4 q;
        uint16_t h[8];
        uint32_t w[4];
    } u;
    u.q = attn_u32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < N - 1; ++i) {
        if (e + i >= n) break;
        if constexpr (DT == SDGP_BF16) u.h[i] = reinterpret_cast<const uint16_t*>(row)[e + i];
        else u.w[i] = reinterpret_cast<const uint32_t*>(row)[e + i];
    }
    return u.q;
}

// Eight values from element e on, as an operand.
template <int DT>
__device__ __forceinline__ Operand<DT> load_operand(const char* row, int e, int n) {
    Operand<DT> f;
    if constexpr (DT == SDGP_BF16) {
        f.w = load_chunk<DT>(row, e, n);
    } else {
        const attn_u32x4 a = load_chunk<DT>(row, e, n), b = load_chunk<DT>(row, e + 4, n);
#pragma unroll
        for (int i = 0; i < 4; ++i) f.x[i] = bits_to_float(a[i]), f.x[4 + i] = bits_to_float(b[i]);
    }
    return f;
}

// The same of rows of whole chunks on sixteen bytes.
template <int DT, bool FAST>
__device__ __forceinline__ Operand<DT> load_operand(const char* row, int e, int n) {
    if constexpr (!FAST) return load_operand<DT>(row, e, n);
    constexpr int N = 16 / Operand<DT>::kSize;                          // an operand is 8 / N chunks
    union {
        Operand<DT> f;
        attn_u32x4 w[8 / N];
    } u;
#pragma unroll
    for (int i = 0; i < 8 / N; ++i) {
        u.w[i] = attn_u32x4{0, 0, 0, 0};
        if (e + i * N < n) u.w[i] = *reinterpret_cast<const attn_u32x4*>(row + (e + i * N) * Operand<DT>::kSize);
    }
    return u.f;
}

// A tile of rows of up to DC values in LDS.  Its sixteen-byte chunks change places within a row (XOR with a number of the
// row) so that both ways of reading it meet all banks: `rows`, sixteen lanes at one chunk of sixteen rows; `columns`, four
// rows of four neighbouring chunks.
template <int DT, int DC>
struct Tile {
    static constexpr int kRow = (DC <= 64 ? 64 : 128) * Operand<DT>::kSize;   // bytes
    static constexpr int kChunks = kRow / 16;

    static __device__ __forceinline__ int place(int row) {
        return kChunks == 8 ? ((row & 2) << 1 | ((row >> 2) & 3)) : ((row & 3) << 2 | ((row >> 2) & 3));
    }
    static __device__ __forceinline__ int at(int row, int chunk) { return row * kRow + ((chunk ^ place(row)) << 4); }

    // A lane's place in a tile, for `rows` and for `columns`.  Which chunk and which block of columns comes last into an address, as
    // an XOR of its lower bits: the one register serves every read of the tile.  Tiles begin on a multiple of a row.
    static __device__ __forceinline__ uint32_t rows_lane(SDGP_SHARED char* tile, int lane) {
        return (uint32_t)(uintptr_t)tile + (uint32_t)at(lane & 31, (lane >> 5) * (DT == SDGP_BF16 ? 1 : 2));
    }
    static __device__ __forceinline__ uint32_t columns_lane(SDGP_SHARED char* tile, int lane) {
        if constexpr (DT == SDGP_BF16)   // of sixteen lanes, each four on one row: the transposing read hands lane i column i of the four rows
            return (uint32_t)(uintptr_t)tile + (uint32_t)(at(4 * (lane >> 5) + ((lane & 15) >> 2), ((lane >> 3) & 2) + ((lane & 3) >> 1)) + (lane & 1) * 8);
        return (uint32_t)(uintptr_t)tile + (uint32_t)(at(4 * (lane >> 5), (lane & 31) >> 2) + (lane & 3) * 4);
    }

    // Rows r0 + lane % 32 of the tile `plus` bytes on, values 16 step + 8 (lane / 32) ..: an operand summed over the values.  r0 % 32 == 0.
    static __device__ __forceinline__ Operand<DT> rows(uint32_t lane_at, int r0, int step, int plus = 0) {
        Operand<DT> f;
        if constexpr (DT == SDGP_BF16) {
            f.w = *(SDGP_SHARED attn_u32x4*)(uintptr_t)((lane_at ^ (uint32_t)(step << 5)) + (uint32_t)(r0 * kRow + plus));
        } else {
            const attn_u32x4 a = *(SDGP_SHARED attn_u32x4*)(uintptr_t)((lane_at ^ (uint32_t)(step << 6)) + (uint32_t)(r0 * kRow + plus));
            const attn_u32x4 b = *(SDGP_SHARED attn_u32x4*)(uintptr_t)((lane_at ^ (uint32_t)(step << 6 | 16)) + (uint32_t)(r0 * kRow + plus));
#pragma unroll
            for (int i = 0; i < 4; ++i) f.x[i] = bits_to_float(a[i]), f.x[4 + i] = bits_to_float(b[i]);
        }
        return f;
    }

    // Column 32 block + lane % 32 of rows r0 + result_row(0 .. 7, lane / 32): an operand summed over the rows, its eight in the
    // order in which a lane holds half a result's rows, so that results are the other operand as they are.  r0 % 16 == 0.
    static __device__ __forceinline__ Operand<DT> columns(uint32_t lane_at, int r0, int block, int plus = 0) {
        Operand<DT> f;
        if constexpr (DT == SDGP_BF16) {
            attn_s16x4 x[2];
#pragma unroll
            for (int u = 0; u < 2; ++u)                                 // eight rows on, `place` differs by two
                x[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (SDGP_SHARED attn_s16x4*)(uintptr_t)((lane_at ^ (uint32_t)(block << 6 | u << 5)) + (uint32_t)((r0 + 8 * u) * kRow + plus)));
            const attn_s16x8 all = {x[0][0], x[0][1], x[0][2], x[0][3], x[1][0], x[1][1], x[1][2], x[1][3]};
            f.w = __builtin_bit_cast(attn_u32x4, all);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {                               // row i % 4 + 8 (i / 4) of the lane's four
                static_assert(kChunks >= 16, "fp32 rows");
                const uint32_t places = (uint32_t)((i & 3) << 2 | (i >> 2) << 1);
                f.x[i] = *(SDGP_SHARED float*)(uintptr_t)((lane_at ^ ((uint32_t)(block << 7) ^ places << 4)) + (uint32_t)((r0 + (i & 3) + 8 * (i >> 2)) * kRow + plus));
            }
        }
        return f;
    }
};

// A value that the compiler computes where it stands and not ahead of a loop: registers are worth more there.
__device__ __forceinline__ uint32_t here(uint32_t x) {
    asm volatile("" : "+v"(x));
    return x;
}

// Buffer loads straight into LDS, lane i's bytes at `lds` + SIZE i; offsets from kNoRecord on give zeros.  The compiler does not count
// them: nothing that it waits for may be on its way beside them, or its wait is for them too.  Nor does it keep the five wait states between
// a vector instruction that writes a scalar register (`records` makes some) and a memory instruction that reads it: s_mov_b32 and s_nop 3 do.
constexpr uint32_t kNoRecord = 0x7FFFFFF0u;

__device__ __forceinline__ attn_u32x4 records(const void* base, uint32_t bytes) {
    const uint64_t at = (uint64_t)(uintptr_t)base;
    attn_u32x4 v;
    v[0] = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at);
    v[1] = (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(at >> 32) & 0xFFFFu));
    v[2] = (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes);
    v[3] = 0x00027000u;
    return v;
}
template <int SIZE>
__device__ __forceinline__ void copy_to_lds(attn_u32x4 from, uint32_t offset, uint32_t lds) {
    static_assert(SIZE == 16 || SIZE == 4, "bytes a lane");
    if constexpr (SIZE == 16) asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(from) : "memory");
    else asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(from) : "memory");
}
__device__ __forceinline__ void wait_for_copies() { __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8)); }   // vmcnt 0

// Where this wavefront's part of each 4096 bytes that 256 threads copy goes.
__device__ __forceinline__ uint32_t wave_part(SDGP_SHARED char* tile) {
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(uintptr_t)tile + (threadIdx.x / 64 << 10)));
}

// Brings rows of a tensor into a tile while the one before it is worked on: `start` asks for them, `finish` comes before the
// barrier behind which they are read.  256 threads; ROWS rows of up to DC values, zeros behind the tensor's last row.
//
// FAST: straight into LDS (buffer loads, whose bounds check makes the zeros), sixteen bytes a lane, each lane the chunk that belongs
// where its bytes land.  Rows on sixteen bytes, D a whole number of chunks.  Else by way of registers, from any element on.
template <int DT, int DC, int ROWS, bool FAST>
struct Feed;

template <int DT, int DC, int ROWS>
struct Feed<DT, DC, ROWS, true> {
    using T = Tile<DT, DC>;
    static constexpr int kEach = ROWS * T::kChunks / 256;               // instructions a wavefront
    static constexpr int kStep = 256 / T::kChunks;                      // rows between them
    static constexpr int kPlaces = kStep % 16 == 0 ? 1 : 2;             // `place` tells sixteen rows apart
    static_assert(kEach * 256 == ROWS * T::kChunks && kStep * kPlaces % 16 == 0, "whole instructions");
    const char* base;
    int64_t row;
    int width;
    uint32_t first[kPlaces];

    __device__ __forceinline__ Feed(const char* tensor, int64_t row_bytes, int D) : base(tensor), row(row_bytes), width(D * Operand<DT>::kSize) {
#pragma unroll
        for (int i = 0; i < kPlaces; ++i) {
            const int r = (int)threadIdx.x / T::kChunks + i * kStep, chunk = ((int)threadIdx.x % T::kChunks) ^ T::place(r);
            first[i] = chunk * 16 < width ? (uint32_t)(r * (int)row_bytes + chunk * 16) : kNoRecord;
        }
    }
    // rows r0 .. r0 + ROWS - 1 of `rows`
    __device__ __forceinline__ void start(SDGP_SHARED char* tile, int r0, int rows) {
        const int64_t left = (int64_t)(rows - r0 - 1) * row + width;
        const attn_u32x4 from = records(base + r0 * row, rows <= r0 ? 0 : left < kNoRecord ? (uint32_t)left : kNoRecord);
        const uint32_t lds = wave_part(tile);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t at = first[i % kPlaces];
            copy_to_lds<16>(from, at == kNoRecord ? at : at + (uint32_t)(i / kPlaces * kPlaces * kStep) * (uint32_t)row, lds + i * 4096);
        }
    }
    __device__ __forceinline__ void finish(SDGP_SHARED char*) { wait_for_copies(); }
};

template <int DT, int DC, int ROWS>
struct Feed<DT, DC, ROWS, false> {
    using T = Tile<DT, DC>;
    static constexpr int kNeed = DC * Operand<DT>::kSize / 16;          // chunks of a row that anyone reads
    static constexpr int kEach = ROWS * T::kChunks / 256;
    attn_u32x4 held[kEach];
    const char* base;
    int64_t row;
    int D;

    __device__ __forceinline__ Feed(const char* tensor, int64_t row_bytes, int width) : base(tensor), row(row_bytes), D(width) {}
    __device__ __forceinline__ void start(SDGP_SHARED char*, int r0, int rows) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int x = (int)threadIdx.x + i * 256, r = x / T::kChunks, chunk = x % T::kChunks;
            held[i] = attn_u32x4{0, 0, 0, 0};
            if (chunk < kNeed && r0 + r < rows) held[i] = load_chunk<DT>(base + (r0 + r) * row, chunk * (16 / Operand<DT>::kSize), D);
        }
    }
    __device__ __forceinline__ void finish(SDGP_SHARED char* tile) const {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int x = (int)threadIdx.x + i * 256, r = x / T::kChunks, chunk = x % T::kChunks;
            if (chunk < kNeed) *(SDGP_SHARED attn_u32x4*)(tile + T::at(r, chunk)) = held[i];
        }
    }
};

// The same of queries: a tile is `tokens` tokens times `heads` heads of a group, head by head (as many as its rows hold).
template <int DT, int DC, int ROWS, bool FAST>
struct FeedQueries {
    using T = Tile<DT, DC>;
    static constexpr int kNeed = DC * Operand<DT>::kSize / 16, kEach = ROWS * T::kChunks / 256, kStep = 256 / T::kChunks;
    attn_u32x4 held[FAST ? 1 : kEach];
    const char* base;                                                   // of the tile that is asked for next
    int64_t row, head;
    int D;

    __device__ __forceinline__ FeedQueries(const char* tensor, int64_t token_bytes, int64_t head_bytes, int width)
        : base(tensor), row(token_bytes), head(head_bytes), D(width) {}
    // `tokens` and `heads` of those are there
    __device__ __forceinline__ void start(SDGP_SHARED char* tile, FastDiv by_heads, int per, int tokens, int heads) {
        const int r0 = (int)threadIdx.x / T::kChunks, at = (int)threadIdx.x % T::kChunks;
        if constexpr (FAST) {
            const attn_u32x4 from = records(base, kNoRecord);
            const uint32_t lds = wave_part(tile);
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int r = r0 + i * kStep, chunk = at ^ T::place(r), t = (int)divide((uint32_t)r, by_heads), g = r - t * per;
                const bool there = t < tokens && g < heads && chunk * 16 < D * Operand<DT>::kSize;
                copy_to_lds<16>(from, there ? (uint32_t)t * (uint32_t)row + (uint32_t)g * (uint32_t)head + (uint32_t)chunk * 16u : kNoRecord, lds + i * 4096);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int r = r0 + i * kStep, t = (int)divide((uint32_t)r, by_heads), g = r - t * per;
                held[i] = attn_u32x4{0, 0, 0, 0};
                if (at < kNeed && t < tokens && g < heads) held[i] = load_chunk<DT>(base + t * row + g * head, at * (16 / Operand<DT>::kSize), D);
            }
        }
    }
    __device__ __forceinline__ void finish(SDGP_SHARED char* tile) const {
        if constexpr (FAST) {
            wait_for_copies();
        } else {
            const int r0 = (int)threadIdx.x / T::kChunks, at = (int)threadIdx.x % T::kChunks;
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (at < kNeed) *(SDGP_SHARED attn_u32x4*)(tile + T::at(r0 + i * kStep, at)) = held[i];
        }
    }
};

// The larger and the sum of a lane's value and that of the lane 32 away.
__device__ __forceinline__ float halves_max(float x) { return fmaxf(x, __shfl_xor(x, 32)); }
__device__ __forceinline__ float halves_sum(float x) { return x + __shfl_xor(x, 32); }

// Stores a 32-column block of results, transposed: lane % 32 is a row of memory, the result's rows its values.
// FAST: D is a whole number of chunks, rows on sixteen bytes.
template <int DT, bool FAST = false>
__device__ __forceinline__ void store_block(char* row, const attn_f32x16& x, int block, int half, int D, float factor) {
    if constexpr (FAST) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int e = 32 * block + 8 * g + 4 * half;
            if (e >= D) break;
            const float y[4] = {x[4 * g] * factor, x[4 * g + 1] * factor, x[4 * g + 2] * factor, x[4 * g + 3] * factor};
            if constexpr (DT == SDGP_BF16) {
                typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
                *reinterpret_cast<u32x2*>(row + e * 2) = u32x2{float2_to_bf16x2(y[0], y[1]), float2_to_bf16x2(y[2], y[3])};
            } else {
                typedef float f32x4 __attribute__((ext_vector_type(4)));
                *reinterpret_cast<f32x4*>(row + e * 4) = f32x4{y[0], y[1], y[2], y[3]};
            }
        }
        return;
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int e = 32 * block + 8 * g + 4 * half;
        const float y[4] = {x[4 * g] * factor, x[4 * g + 1] * factor, x[4 * g + 2] * factor, x[4 * g + 3] * factor};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (DT == SDGP_BF16) {
                if (i & 1) continue;
                const uint32_t w = float2_to_bf16x2(y[i], y[i + 1]);
                uint16_t* p = reinterpret_cast<uint16_t*>(row) + e + i;
                if (e + i + 1 < D) {
                    typedef uint32_t word_half __attribute__((aligned(2), may_alias));
                    *reinterpret_cast<word_half*>(p) = w;
                } else if (e + i < D) {
                    *p = (uint16_t)w;
                }
            } else if (e + i < D) {
                reinterpret_cast<float*>(row)[e + i] = y[i];
            }
        }
    }
}

}  // namespace sdgp
