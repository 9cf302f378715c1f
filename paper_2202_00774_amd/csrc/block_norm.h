// Arguments of the block norms' kernels and how their backward pass cuts the rows into slabs.
#pragma once

#include "rows.h"

namespace sdgp {

struct Norm {
    const void *x, *u, *gate, *w_post, *w_pre;
    void *y, *h;
    float* stats;
    int64_t rows, per_gate;   // rows that share a gate
    int D, dt, wdt;
    float residual_scale, eps;
};

// The rows of a slab belong to one workgroup, which keeps its columns' sums in registers and leaves them in the workspace.
// Two ways to cut: kInGroup, `parts` slabs of `len` rows for every gate (one "gate" for all rows where there is none),
// the sums of dY a of a slab then being a gate's; kWholeGroups, `len` gates a slab, where gates of few rows are many: the
// slab finishes its gates itself.
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
};

// Threads a row and 16-byte vectors a thread, for rows that fit the registers: 16 lanes for the narrowest, a wavefront,
// then 256 to 1024 threads.  0 threads: the row is longer (above 16384 bf16 or 8192 fp32 values).
struct RowShape {
    int threads, vecs;
};

inline RowShape row_shape(int64_t D, int dt) {
    const int64_t vecs = (D + (dt == SDGP_BF16 ? 7 : 3)) / (dt == SDGP_BF16 ? 8 : 4);
    for (const RowShape s : {RowShape{16, 1}, {16, 2}, {64, 1}, {64, 2}, {256, 1}, {256, 2}, {512, 2}, {1024, 2}})
        if (vecs <= s.threads * s.vecs) return s;
    return {0, 0};
}

template <int DT>
int norm_rows_launch(const Norm& n, RowShape shape, hipStream_t stream);
template <int DT>
int norm_grad_launch(const NormGrad& n, RowShape shape, hipStream_t stream);

}  // namespace sdgp
