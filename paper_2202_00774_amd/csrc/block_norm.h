// Arguments of the block norms' kernels and how their backward pass cuts the rows into slabs.
#pragma once

#include <initializer_list>

#include "rows.h"

namespace sdgp {

struct Norm {
    const void *x, *u, *gate, *w_post, *w_pre;
    void *y, *h;
    float* stats;
    int64_t rows, per_gate;   // rows that share a gate
    int D, dt, wdt;
    float residual_scale, eps;
    bool aligned, large;
};

// The rows of a slab belong to one workgroup, which keeps its columns' sums in registers and leaves them in the workspace.
// Two ways to cut: kInGroup, `parts` slabs of `len` rows for every gate (one "gate" for all rows where there is none),
// the sums of dY a of a slab then being a gate's; kWholeGroups, `len` gates a slab, where gates of few rows are many: the
// slab finishes its gates itself.  Slabs in a gate are consecutive rows, or, in large tensors, every parts-th of the rows
// that are worked on at a time, so that all workgroups together walk through memory in one front.
enum SlabKind { kInGroup, kWholeGroups };

struct Slabs {
    SlabKind kind;
    int64_t count, parts, len;
};

struct NormGrad {
    const void *dy, *dh, *y, *u, *gate, *w_post, *w_pre;
    const float* stats;
    void *dx, *du, *dgate;
    float *dw_post, *dw_pre;
    float *part_pre, *part_post;   // [slabs, D]
    int64_t rows, groups, per_gate;
    Slabs slabs;
    int D, dt, wdt;
    float residual_scale;
    bool aligned, large;
};

// Rows that begin on 16 bytes are read with the streaming hint (55 -> 50 us forward, 16384 x 2048 bf16); others share lines
// between neighbouring loads, which the hint would fetch twice (35 -> 51 us backward, 4099 x 1001 fp32).
inline bool rows_aligned(int64_t D, int dt, std::initializer_list<const void*> tensors) {
    uintptr_t a = (uintptr_t)(D * (dt == SDGP_BF16 ? 2 : 4));
    for (const void* p : tensors) a |= reinterpret_cast<uintptr_t>(p);
    return (a & 15u) == 0;
}

// Tensors that leave nothing in the last-level cache (256 MB, for two results and the gradients that come next) are written
// with the streaming hint, and workgroups take rows in turn instead of slabs in one piece.  Forward and backward together,
// slabs and plain stores against turns and streaming ones: 130 / 146 us at 16384 x 2048 bf16 (67 MB), 561 / 484 at
// 32768 x 4096 (268 MB).
inline bool rows_large(int64_t rows, int64_t D, int dt) { return rows * D * (dt == SDGP_BF16 ? 2 : 4) > ((int64_t)128 << 20); }

// Threads a row and 16-byte vectors a thread, for rows that fit the registers: one vector each, from 16 lanes to 1024
// threads, two above that.  Loads in flight bound these kernels, so idle lanes count: with 192, 384 and 768 threads beside the
// powers of two 30000 x 1104 bf16 takes 169 us instead of 190, 16384 x 2560 156 instead of 172, both directions.  (Two vectors
// and half the threads: 331 us against 301 at 8192 x 8192, 92 against 77 at 4096 x 4096.)  0 threads: the row is longer (above
// 16384 bf16 or 8192 fp32 values).
struct RowShape {
    int threads, vecs;
};

// Rows that a workgroup (of 256 threads, or a row's) works on at a time.
constexpr int rows_at_once(int threads) { return threads < 192 ? 256 / threads : 1; }

inline RowShape row_shape(int64_t D, int dt) {
    const int64_t vecs = (D + (dt == SDGP_BF16 ? 7 : 3)) / (dt == SDGP_BF16 ? 8 : 4);
    for (const RowShape s : {RowShape{16, 1}, {32, 1}, {64, 1}, {128, 1}, {192, 1}, {256, 1}, {384, 1}, {512, 1}, {768, 1}, {1024, 1}, {1024, 2}})
        if (vecs <= s.threads * s.vecs) return s;
    return {0, 0};
}

template <int DT>
int norm_rows_launch(const Norm& n, RowShape shape, hipStream_t stream);
template <int DT>
int norm_grad_launch(const NormGrad& n, RowShape shape, hipStream_t stream);

}  // namespace sdgp
