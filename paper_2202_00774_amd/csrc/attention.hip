// Which attention kernels a call takes, and the room its pieces need.
//
// The forward pass gives 128 rows (query tokens times heads of a group) to a workgroup, or 32 rows to four wavefronts that split
// the keys, where sequences have few rows (single tokens).  Where that leaves the chip short of workgroups the keys are cut into up
// to 64 parts, whose sums a second kernel joins.
#include <math.h>

#include "attention.h"
#include "attention_api.h"

namespace sdgp {

template <int DT>
int attention_fwd_launch(const Attention& a, int64_t tiles, bool few, hipStream_t stream);
template <int DT>
int attention_bwd_launch(Attention a, const AttentionGrid& g, hipStream_t stream);

namespace {

constexpr int64_t kMostWorkgroups = 0xFFFFFF;   // of 256 threads: a launch counts threads in 32 bits

struct Split {
    bool few;
    int parts;
};

// By the sequences' mean lengths: of packed ones the host knows no more.
Split choose(int64_t S, int64_t Tq, int64_t Tk, int64_t H, int64_t Hk) {
    const int64_t n = S > 0 ? S : 1, rows = (Tq + n - 1) / n * (H / Hk), keys = (Tk + n - 1) / n;
    Split s;
    s.few = rows <= 32;
    const int64_t unit = s.few ? 32 : 128, groups = n * ((rows + unit - 1) / unit) * Hk;
    int64_t parts = groups > 0 ? (s.few ? 1536 : 512) / groups : 1;
    const int64_t most = keys / 128;
    parts = parts > most ? most : parts;
    s.parts = (int)(parts < 1 ? 1 : parts > 64 ? 64 : parts);
    return s;
}

struct BwdSplit {
    int own_rows, parts;
};

BwdSplit choose_bwd(int64_t S, int64_t Tq, int64_t Tk, int64_t H, int64_t Hk, int dt) {
    const int64_t n = S > 0 ? S : 1, tokens = (Tq + n - 1) / n, rows = tokens * (H / Hk), keys = (Tk + n - 1) / n;
    const auto groups = [&](int64_t length, int64_t unit) { return n * ((length + unit - 1) / unit) * Hk; };
    BwdSplit s;
    s.own_rows = groups(rows, 128) >= 512 ? 4 : 2;
    const int64_t have = groups(keys, 32 * attention_own_keys(dt)), rounds = (tokens + 63) / 64 * (H / Hk);
    // Parts cost their sums, written and read, and their own first copies.  8192 tokens, 256 workgroups: 618 us and 23 for the sums in
    // four parts, 590 and 36 in six; 4096 tokens, 64 workgroups: 99 and 12 in eight, 95 and 22 in sixteen; twice 2000 tokens, 128
    // workgroups of D = 64: 23 and 7 in four, 31 and 12 in eight; 1024 tokens, 64 workgroups: 24 and 7 in four (the limit by rounds), 29
    // and 6 in two.  22294 packed tokens, 736 workgroups: a pass takes 1465 us with one part and 1463 with two, at the power the card has.
    int64_t parts = have > 0 ? (dt == SDGP_BF16 && have >= 256 ? 1024 : 512) / have : 1;
    parts = parts > rounds / 4 ? rounds / 4 : parts;
    s.parts = (int)(parts < 1 ? 1 : parts > 16 ? 16 : parts);
    return s;
}

Attention arguments(const AttentionCall& c) {
    Attention a = {};
    a.q = c.q, a.k = c.k, a.v = c.v;
    a.q_token = c.strides[0], a.q_head = c.strides[1], a.k_token = c.strides[2], a.k_head = c.strides[3], a.v_token = c.strides[4], a.v_head = c.strides[5];
    a.off_q = c.offsets_q, a.off_k = c.offsets_k, a.len_k = c.lengths_k;
    a.S = (int)c.S, a.Tq = (int)c.Tq, a.Tk = (int)c.Tk, a.H = (int)c.H, a.Hk = (int)c.Hk, a.G = (int)(c.H / c.Hk), a.D = c.D, a.causal = c.causal;
    a.Lq = c.S > 0 ? (int)(c.Tq / c.S) : 0, a.Lk = c.S > 0 ? (int)(c.Tk / c.S) : 0;
    a.by_group = fast_div((uint32_t)a.G);
    a.scale = c.scale, a.c = c.scale * 1.44269504088896341f;
    a.parts = 1;
    a.buckets = 1;
    // Feed<..., FAST>: whole chunks on sixteen bytes, a token's distance of at least a head and within what a tile's offsets count
    const int64_t size = c.dt == SDGP_BF16 ? 2 : 4;
    uintptr_t all = reinterpret_cast<uintptr_t>(c.q) | reinterpret_cast<uintptr_t>(c.k) | reinterpret_cast<uintptr_t>(c.v) | (uintptr_t)(c.D * size);
    a.fast = true;
    for (int i = 0; i < 6; ++i) {
        all |= (uintptr_t)(c.strides[i] * size);
        if (c.strides[i] * size >= 1 << 23 || (i % 2 == 0 && c.strides[i] < c.D)) a.fast = false;
    }
    a.fast = a.fast && (all & 15u) == 0 && c.H * c.D * size < 1 << 23;
    return a;
}

}  // namespace

// Workgroups by the work they have, where there are more of them than run at once and sequences long enough to differ (finding
// their place takes them up to 8 us).
static int in_order_of_work(const AttentionCall& c, int64_t workgroups) {
    return c.offsets_q != nullptr && c.S > 1 && c.S <= kInOrder && workgroups > 512 && c.Tq >= 512 * c.S ? 4 : 1;
}

size_t attention_workspace(int64_t S, int64_t Tq, int64_t Tk, int64_t H, int64_t Hk, int D) {
    const Split s = choose(S, Tq, Tk, H, Hk);
    return s.parts == 1 ? 0 : (size_t)s.parts * (size_t)(Tq * H) * (size_t)(D + 2) * sizeof(float);
}

size_t attention_bwd_workspace(int64_t S, int64_t Tq, int64_t Tk, int64_t H, int64_t Hk, int D, int dt) {
    const BwdSplit s = choose_bwd(S, Tq, Tk, H, Hk, dt);
    const size_t rows = 2 * (size_t)((Tq * H + 3) / 4 * 4);
    return (rows + (s.parts == 1 ? 0 : (size_t)s.parts * 2 * (size_t)(Tk * Hk) * (size_t)D)) * sizeof(float);
}

int attention_launch(const AttentionCall& c, void* o, float* lse, void* workspace, hipStream_t stream) {
    Attention a = arguments(c);
    const Split s = choose(c.S, c.Tq, c.Tk, c.H, c.Hk);
    a.o = o, a.lse = lse, a.parts = s.parts;
    a.fast = a.fast && (reinterpret_cast<uintptr_t>(o) & 15u) == 0;
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = a.part_o + (s.parts == 1 ? 0 : (int64_t)s.parts * c.Tq * c.H * c.D);
    const int64_t tiles = most_tiles(c.offsets_q != nullptr, c.S, c.Tq, a.Lq, a.G, s.few ? 32 : 128);
    if (tiles * a.Hk * a.parts > kMostWorkgroups) return SDGP_ERR_SHAPE;
    a.buckets = in_order_of_work(c, tiles * a.Hk * a.parts);
    return c.dt == SDGP_BF16 ? attention_fwd_launch<SDGP_BF16>(a, tiles, s.few, stream) : attention_fwd_launch<SDGP_F32>(a, tiles, s.few, stream);
}

int attention_bwd_launch_all(const AttentionCall& c, const void* d_o, const void* o, const float* lse, void* dq, void* dk, void* dv,
                             void* workspace, hipStream_t stream) {
    Attention a = arguments(c);
    a.d_o = d_o, a.o_in = o, a.lse = const_cast<float*>(lse), a.dq = dq, a.dk = dk, a.dv = dv;
    a.lse2 = static_cast<float*>(workspace);
    a.delta = a.lse2 + (c.Tq * c.H + 3) / 4 * 4;
    for (const void* p : {d_o, o, (const void*)dq, (const void*)dk, (const void*)dv}) a.fast = a.fast && (reinterpret_cast<uintptr_t>(p) & 15u) == 0;
    const bool packed = c.offsets_q != nullptr;
    const BwdSplit s = choose_bwd(c.S, c.Tq, c.Tk, c.H, c.Hk, c.dt);
    a.parts = s.parts;
    a.part_o = a.delta + (c.Tq * c.H + 3) / 4 * 4;
    const int rows = attention_dkv_rows(c.dt, a.fast ? (c.D <= 64 ? 64 : c.D <= 96 ? 96 : 128) : 128, attention_own_keys(c.dt));
    a.by_heads = fast_div((uint32_t)(a.G < rows ? a.G : rows));
    AttentionGrid g;
    g.own_rows = s.own_rows;
    g.row_tiles = c.Tq == 0 ? 0 : most_tiles(packed, c.S, c.Tq, a.Lq, a.G, 32 * s.own_rows);
    g.key_tiles = c.Tk == 0 ? 0 : most_tiles(packed, c.S, c.Tk, a.Lk, 1, 32 * attention_own_keys(c.dt));
    a.buckets = in_order_of_work(c, g.key_tiles * a.Hk * a.parts);
    if (g.row_tiles * a.Hk > kMostWorkgroups || g.key_tiles * a.Hk * a.parts > kMostWorkgroups) return SDGP_ERR_SHAPE;
    return c.dt == SDGP_BF16 ? attention_bwd_launch<SDGP_BF16>(a, g, stream) : attention_bwd_launch<SDGP_F32>(a, g, stream);
}

}  // namespace sdgp
