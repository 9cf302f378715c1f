// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and their gradient.
//
//   z = scale * x;  m = max x;  s = sum_j e^(z_j - scale m)
//   logp = (x_t - m) scale - ln s        entropy = ln s - (1/s) sum_j e^(z_j - scale m) (z_j - scale m)
//   dL/dx_j = scale * (g (d_jt - p_j) - h p_j (ln p_j + entropy)),  g = dL/dlogp, h = dL/dentropy
//
// One pass over a row: running maximum, sum and weighted sum, and the best `top` logits so far.  A wavefront has one maximum
// for all its lanes; only when a chunk brings a larger one (a few times a row) are its sums brought to it.  Differences to
// the maximum are taken before the scale is applied, so a mask of the type's lowest value cannot overflow into a NaN; in the
// weighted sum they are cut at -256 (in powers of two), where e^ is 0 already, so that a logit of -inf adds 0 and not
// 0 * inf.  All sums are fp32.
//
// Bound by memory where rows are many: 2 bytes an element read forward, 4 read and written backward in bf16, with 8 vector
// instructions beside them forward, 10 backward and 12 with the entropy's gradient, one an exponential.  A row is one workgroup's (or, where rows are short and many, one
// wavefront's); few long rows are cut into pieces, whose sums and lists a second kernel joins.  Measured: 8192 x 65536 bf16
// forward 169 us (6.4 TB/s), gradient 355 to 361 (6.0 TB/s); 4 x 131072 with eight alternatives 9 + 5 us, which are latencies.
#include "rows.h"

namespace sdgp {

namespace {

constexpr int kBlock = 256, kWave = 64;
constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kFloor2 = -256.0f;   // exponents of two below this count as this: 2^-256 is 0 in fp32
constexpr int kMaxTop = 64;          // a wavefront keeps its best logits one a lane

// 2^x by the one instruction: good to a unit in the last place, and 0 below 2^-126.  So a probability that small counts as 0: beside
// the row's largest term, which is 1, that is nothing; in the gradient it is what the type hardly holds.
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// max, sum of 2^(c (x - max)), sum of 2^(c (x - max)) * c (x - max)
struct Sums {
    float m, s, a;
};

__device__ __forceinline__ float exponent(float x, float m, float c) { return (x - m) * c; }

// The sums as they are with the maximum m >= t.m.
__device__ __forceinline__ void rebase(Sums& t, float m, float c) {
    const float d = fmaxf(exponent(t.m, m, c), kFloor2), f = exp2_hw(d);
    t.a = f * (t.a + t.s * d);
    t.s *= f;
    t.m = m;
}

__device__ __forceinline__ Sums joined(Sums p, Sums q, float c) {
    const float m = fmaxf(p.m, q.m);
    rebase(p, m, c);
    rebase(q, m, c);
    return {m, p.s + q.s, p.a + q.a};
}

template <int DT>
__device__ __forceinline__ float load_logit(const void* row, int64_t j) {
    if constexpr (DT == SDGP_BF16) return bf16_to_float(static_cast<const uint16_t*>(row)[j]);
    else return static_cast<const float*>(row)[j];
}

template <int DT>
constexpr uint32_t kMinusInf = DT == SDGP_BF16 ? 0xFF80FF80u : 0xFF800000u;

// Largest over the wavefront, the same for all lanes.
__device__ __forceinline__ float max64(float v) {
    v = fmaxf(v, lane_swap<0xB1>(v));
    v = fmaxf(v, lane_swap<0x4E>(v));
    v = fmaxf(v, lane_swap<0x141>(v));
    v = fmaxf(v, lane_swap<0x140>(v));
    return fmaxf(fmaxf(lane_value(v, 0), lane_value(v, 16)), fmaxf(lane_value(v, 32), lane_value(v, 48)));
}

// The best logits a wavefront has met, lane i the i-th; equal logits in the order of their index.  Places not taken
// hold -inf and the index -1 (as unsigned the largest).
struct Best {
    float x;
    uint32_t j;
};

__device__ __forceinline__ bool better(float x, uint32_t j, float y, uint32_t k) { return x > y || (x == y && j < k); }

__device__ __forceinline__ uint32_t from_lane_below(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x138, 0xF, 0xF, false);   // wave_shr 1; lane 0 keeps its own
}

// Takes one logit (the same for all lanes) into the list: the ones it is better than move up a lane.
__device__ __forceinline__ void insert(Best& b, float x, uint32_t j) {
    const bool keep = better(b.x, b.j, x, j);
    const float ux = bits_to_float(from_lane_below(float_to_bits(b.x)));
    const uint32_t uj = from_lane_below(b.j);
    const bool moves = (threadIdx.x & (kWave - 1)) != 0 && !better(ux, uj, x, j);   // the one below moves up to here
    if (!keep) {
        b.x = moves ? ux : x;
        b.j = moves ? uj : j;
    }
}

__device__ __forceinline__ uint32_t lane_word(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }

// The value of lane (own ^ X), without the LDS: within 16 lanes by DPP (4 as 7 and 3), between rows and halves by the swaps.
template <int X>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
    constexpr int kDpp = X == 1 ? 0xB1 : X == 2 ? 0x4E : X == 3 ? 0x1B : X == 7 ? 0x141 : X == 15 ? 0x140 : X == 8 ? 0x128 : 0;
    if constexpr (kDpp != 0) {
        return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kDpp, 0xF, 0xF, true);
    } else if constexpr (X == 4) {
        return lane_xor<3>(lane_xor<7>(v));
    } else if constexpr (X == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);   // rows 0 0 2 2 and 1 1 3 3
        return (threadIdx.x & 16) ? r[0] : r[1];
    } else if constexpr (X == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);   // the lower half twice, the upper half twice
        return (threadIdx.x & 32) ? r[0] : r[1];
    } else if constexpr (X == 31) {
        return lane_xor<15>(lane_xor<16>(v));
    } else {
        static_assert(X == 63, "");
        return lane_xor<31>(lane_xor<32>(v));
    }
}

// Of each pair of lanes l, l ^ X the lower one keeps the better logit.
template <int X>
__device__ __forceinline__ void exchange(Best& b) {
    constexpr int kTop = X >= 32 ? 32 : X >= 16 ? 16 : X >= 8 ? 8 : X >= 4 ? 4 : X >= 2 ? 2 : 1;   // set in the upper of a pair
    const Best o = {bits_to_float(lane_xor<X>(float_to_bits(b.x))), lane_xor<X>(b.j)};
    const bool lower = (threadIdx.x & kTop) == 0;
    if (better(o.x, o.j, b.x, b.j) == lower) b = o;   // equal pairs (two empty places) may swap: they are alike
}

// Sorts one logit a lane, the best first.
__device__ __forceinline__ void sort(Best& b) {
    exchange<1>(b);
    exchange<3>(b), exchange<1>(b);
    exchange<7>(b), exchange<2>(b), exchange<1>(b);
    exchange<15>(b), exchange<4>(b), exchange<2>(b), exchange<1>(b);
    exchange<31>(b), exchange<8>(b), exchange<4>(b), exchange<2>(b), exchange<1>(b);
    exchange<63>(b), exchange<16>(b), exchange<8>(b), exchange<4>(b), exchange<2>(b), exchange<1>(b);
}

// The 64 best of two sorted lists, the second one given from its end: of each pair the better one, then put in order.
__device__ __forceinline__ void merge_reversed(Best& b, const Best& end_first) {
    if (better(end_first.x, end_first.j, b.x, b.j)) b = end_first;
    exchange<32>(b), exchange<16>(b), exchange<8>(b), exchange<4>(b), exchange<2>(b), exchange<1>(b);
}

// Takes in one logit a lane, in any order.
__device__ __forceinline__ void merge_unsorted(Best& b, Best o) {
    sort(o);
    merge_reversed(b, {bits_to_float(lane_xor<63>(float_to_bits(o.x))), lane_xor<63>(o.j)});
}

// What the wavefronts of a row tell each other: how good a logit must at least be.  A row's `top` best are no worse than
// any one wavefront's last, and no worse than the worst of the wavefronts' (top / 4)-th, since these are `top` logits
// together.  Written and read without a barrier: whatever a reader meets was a lower bound when it was written, and is one.
struct Bounds {
    volatile float least, share[kBlock / kWave];

    __device__ __forceinline__ void tell(int wave, float last, float own_share) {
        share[wave] = own_share;
        const float all = fminf(fminf(share[0], share[1]), fminf(share[2], share[3]));
        least = fmaxf(least, fmaxf(last, all));
    }
};

// A bound before there is any list, from each lane's best of the first chunk: in every one of `groups` groups of lanes
// (a power of two, 16 at most) there is a logit that is not less.  With the other wavefronts' it leaves a few logits of the
// first chunk to take in, where else every lane has one (2048 x 50021 bf16 with 4 alternatives 62.5 us without, 57.5 with it).
__device__ __forceinline__ float first_bound(float x, int groups) {
    float m = fmaxf(x, lane_swap<0xB1>(x));
    m = fmaxf(m, lane_swap<0x4E>(m));                        // a quad's best
    if (groups <= 8) m = fmaxf(m, lane_swap<0x141>(m));      // of eight lanes
    if (groups <= 4) m = fmaxf(m, lane_swap<0x140>(m));      // of sixteen
    if (groups > 4) {
        m = fminf(m, lane_swap<0x140>(m));
        if (groups > 8) m = fminf(m, lane_swap<0x141>(m));
    }
    const float a = lane_value(m, 0), b = lane_value(m, 16), c = lane_value(m, 32), d = lane_value(m, 48);
    return groups == 1 ? fmaxf(fmaxf(a, b), fmaxf(c, d)) : groups == 2 ? fminf(fmaxf(a, b), fmaxf(c, d)) : fminf(fminf(a, b), fminf(c, d));
}

// Groups a wavefront that four of them have `top` in all.
__device__ __forceinline__ int share_groups(int top) { return top <= 4 ? 1 : top <= 8 ? 2 : top <= 16 ? 4 : top <= 32 ? 8 : 16; }

constexpr int kOneByOne = 4;   // up to so many lanes with new ones, they go in one by one (25 instructions each); else a
                               // lane's best each together (190)

// Offers the N logits that each lane holds, lane l those of the indexes first + l * N onwards, larger than any index that
// was offered before; `bound`: what is less is not among the best.  A logit like the last in the list is no better than
// it, its index being larger; but among those offered here it may be, so the list's end is compared with its index.
template <int N>
__device__ __forceinline__ void offer(Best& b, int top, float bound, float (&x)[N], float most, uint32_t first) {
    const int lane = threadIdx.x & (kWave - 1);
    const uint32_t j0 = first + (uint32_t)(lane * N);
    uint64_t who = __ballot(most > lane_value(b.x, top - 1) && most >= bound);
    while (who) {
        if (__builtin_popcountll(who) <= kOneByOne) {
            // at least as good as the list's end (one that is only as good may go in behind it), and not -inf
            const float least = fmaxf(fmaxf(lane_value(b.x, top - 1), bound), kLowest);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                uint64_t some = __ballot(x[i] >= least);
                while (some) {
                    const int from = __builtin_ctzll(some);
                    some &= some - 1;
                    insert(b, lane_value(x[i], from), first + (uint32_t)(from * N + i));
                }
            }
            return;
        }
        uint32_t j = 0xFFFFFFFFu;   // a lane's best: the first of equal ones
#pragma unroll
        for (int i = N - 1; i >= 0; --i) j = x[i] == most ? j0 + i : j;
        const bool mine = most >= fmaxf(bound, kLowest) && better(most, j, lane_value(b.x, top - 1), lane_word(b.j, top - 1));
        if (!__ballot(mine)) return;   // each turn takes one away at least
        merge_unsorted(b, {mine ? most : -INFINITY, mine ? j : 0xFFFFFFFFu});
        most = mine ? -INFINITY : most;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (mine && j0 + i == j) x[i] = -INFINITY;
            most = fmaxf(most, x[i]);
        }
        // what is left over may be as good as the list's end, with a lower index
        who = __ballot(most >= fmaxf(fmaxf(lane_value(b.x, top - 1), bound), kLowest));
    }
}

// One wavefront's share of a row, up to element `end`: 64 vectors side by side from element `first` on, kAtOnce of them
// `stride` elements apart in a chunk.  Whole chunks come first, the next one always on its way, then the row's end.
constexpr int kAtOnce = 2;

// Adds a chunk to the sums.  Without a floor under the exponents a masked logit makes the weighted sum a NaN (0 * inf): then
// it is summed again with the floor, and in the row's later chunks at once (`careful`).
template <int N>
__device__ __forceinline__ void add_chunk(Sums& t, const float (&x)[kAtOnce][N], float c, bool& careful) {
    constexpr int M = kAtOnce * N;
    float d[M], p[M], s[2] = {0.0f, 0.0f}, a[2] = {0.0f, 0.0f};   // two chains each
#pragma unroll
    for (int i = 0; i < M; ++i) {
        d[i] = exponent(x[i / N][i % N], t.m, c);
        p[i] = exp2_hw(d[i]);
        s[i & 1] += p[i];
    }
    t.s += s[0] + s[1];
    if (!careful) {
#pragma unroll
        for (int i = 0; i < M; ++i) a[i & 1] = fmaf(p[i], d[i], a[i & 1]);
        a[0] += a[1];
        careful = __ballot(a[0] != a[0]) != 0;
    }
    if (careful) {
        a[0] = a[1] = 0.0f;
#pragma unroll
        for (int i = 0; i < M; ++i) a[i & 1] = fmaf(p[i], fmaxf(d[i], kFloor2), a[i & 1]);
        a[0] += a[1];
    }
    t.a += a[0];
}

template <int DT, bool TOP, Caching LOGITS>
__device__ __forceinline__ void scan(const void* row, int64_t first, int64_t stride, int end, float c, int top, Sums& t, Best& best,
                                     Bounds* bounds, int wave, bool early) {   // early: each of the wavefronts has a whole chunk
    using V = RowVec<DT>;
    constexpr int N = V::kN;
    const int lane = threadIdx.x & (kWave - 1);
    const int64_t step = kAtOnce * stride, span = (kAtOnce - 1) * stride + kWave * N;
    bool careful = false;
    const auto take = [&](const V (&v)[kAtOnce], int64_t e, auto&& then) {
        float x[kAtOnce][N], most[kAtOnce], all = -INFINITY;
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            most[u] = -INFINITY;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                x[u][i] = v[u].get(i);
                most[u] = fmaxf(most[u], x[u][i]);
            }
            all = fmaxf(all, most[u]);
        }
        then();   // the vectors' registers are free
        if (__ballot(all > t.m)) rebase(t, fmaxf(max64(all), t.m), c);
        add_chunk<N>(t, x, c, careful);
        if constexpr (TOP) {
            if (bounds != nullptr && early && e == first) {   // once for every wavefront: there is a barrier
                const float own = first_bound(all, share_groups(top));
                if (lane == 0) bounds->share[wave] = own;
                __syncthreads();
                if (lane == 0) bounds->tell(wave, -INFINITY, own);
            }
            const float bound = bounds != nullptr ? bounds->least : -INFINITY;
            if (__ballot(all > lane_value(best.x, top - 1) && all >= bound)) {
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) offer<N>(best, top, bound, x[u], most[u], (uint32_t)(e + u * stride));
                if (bounds != nullptr) bounds->tell(wave, lane_value(best.x, top - 1), lane_value(best.x, (top + 3) / 4 - 1));
            }
        }
    };

    int64_t e = first;
    V v[kAtOnce];
    if (first + span <= end) {
        const int64_t last = first + (end - first - span) / step * step;   // where the last whole chunk begins
        const auto load = [&](int64_t at) {
            const char* from = static_cast<const char*>(row) + at * (int64_t)sizeof(typename V::Elem);   // the same for all lanes
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u)
                v[u] = load_row<DT, LOGITS>(from + u * stride * (int64_t)sizeof(typename V::Elem), lane * N, INT32_MAX);
        };
        load(e);
        for (; e <= last; e += step)
            take(v, e, [&] { load(e < last ? e + step : last); });
    }
    for (; e < end; e += step) {
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int64_t at = e + u * stride + lane * N;
            v[u] = load_row<DT>(row, (int)(at < end ? at : end), end, kMinusInf<DT>);
        }
        take(v, e, [] {});
    }
    // every lane's sums have the same maximum
    t.s = sum64(t.s);
    t.a = sum64(t.a);
}

struct Logprobs {
    const void *logits, *tokens;
    float *logp, *entropy, *top_logp, *stats;
    int64_t* top_ids;
    int64_t ld, rows;
    int V, top, token_bits;
    float scale;
    // few long rows: pieces of a row, of `piece` elements each, and where their sums and lists go
    int pieces, piece;
    Sums* part_sums;   // [rows, pieces]
    Best* part_best;   // [rows, pieces, top]
    bool stream;
};

// Results of row r from one wavefront's sums and list.
template <int DT>
__device__ __forceinline__ void finish(const Logprobs& q, int64_t r, const Sums& t, const Best& best) {
    const int lane = threadIdx.x & (kWave - 1);
    const float logs = logf(t.s);                    // of an empty row: -inf
    const bool empty = t.s == 0.0f, bad = t.s != t.s;
    if (lane == 0) {
        if (q.logp) {
            const int64_t token = q.token_bits == 64 ? static_cast<const int64_t*>(q.tokens)[r] : (int64_t) static_cast<const int32_t*>(q.tokens)[r];
            const char* row = static_cast<const char*>(q.logits) + r * q.ld * (DT == SDGP_BF16 ? 2 : 4);
            float lp = 0.0f;
            if (token >= q.V) lp = NAN;
            else if (token >= 0) lp = empty ? -INFINITY : (load_logit<DT>(row, token) - t.m) * q.scale - logs;
            q.logp[r] = lp;
        }
        q.entropy[r] = empty ? 0.0f : logs - kLn2 * t.a / t.s;
        q.stats[2 * r] = t.m;
        q.stats[2 * r + 1] = logs;
    }
    if (lane < q.top) {
        const bool none = bad || best.j == 0xFFFFFFFFu;
        q.top_ids[r * q.top + lane] = none ? -1 : (int64_t)best.j;
        q.top_logp[r * q.top + lane] = bad ? NAN : none ? -INFINITY : (best.x - t.m) * q.scale - logs;
    }
}

// The workgroup's sums and list in its first wavefront.
template <bool TOP>
__device__ __forceinline__ void join_waves(Sums& t, Best& best, float c, Sums* part, Best (*lists)[kMaxTop]) {
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    __syncthreads();   // the first wavefront is done with what was there
    if (lane == 0) part[wave] = t;
    if constexpr (TOP) lists[wave][lane] = best;
    __syncthreads();
    if (wave != 0) return;
    for (int w = 1; w < kBlock / kWave; ++w) {
        t = joined(t, part[w], c);
        if constexpr (TOP) merge_reversed(best, lists[w][kWave - 1 - lane]);
    }
}

// T = 64: a wavefront a row; 256: a workgroup a row, or a piece of one.
template <int DT, int T, bool TOP, Caching LOGITS>
__global__ void __launch_bounds__(kBlock) logprob_rows(const Logprobs q) {
    constexpr int N = RowVec<DT>::kN, R = kBlock / T;
    __shared__ Sums part[T > kWave ? kBlock / kWave : 1];
    __shared__ Best lists[T > kWave && TOP ? kBlock / kWave : 1][kMaxTop];
    __shared__ Bounds bounds;
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const float c = q.scale * kLog2e;
    const int64_t items = q.rows * q.pieces;
    for (int64_t i0 = (int64_t)blockIdx.x * R; i0 < items; i0 += (int64_t)gridDim.x * R) {
        const int64_t item = i0 + (T == kWave ? wave : 0);
        if (item >= items) continue;   // T = 64 only, a whole wavefront: nothing is shared
        const int64_t r = item / q.pieces;
        const int begin = (int)(item - r * q.pieces) * q.piece;
        const int end = q.V - begin < q.piece ? q.V : begin + q.piece;
        const char* row = static_cast<const char*>(q.logits) + r * q.ld * (DT == SDGP_BF16 ? 2 : 4);
        Sums t = {kLowest, 0.0f, 0.0f};
        Best best = {-INFINITY, 0xFFFFFFFFu};
        if constexpr (T > kWave && TOP) {
            if (lane == 0) bounds.share[wave] = -INFINITY;
            if (threadIdx.x == 0) bounds.least = -INFINITY;
            __syncthreads();
        }
        scan<DT, TOP, LOGITS>(row, begin + (T == kWave ? 0 : wave * kWave * N), (int64_t)T * N, end, c, q.top, t, best, T > kWave ? &bounds : nullptr, wave,
                              T > kWave && end - begin >= kAtOnce * T * N);
        if constexpr (T > kWave) {
            join_waves<TOP>(t, best, c, part, lists);
            if (wave != 0) continue;
        }
        if (q.pieces == 1) {
            finish<DT>(q, r, t, best);
        } else {
            if (lane == 0) q.part_sums[item] = t;
            if (lane < q.top) q.part_best[item * q.top + lane] = best;
        }
    }
}

// One workgroup a row: each wavefront joins every fourth piece, then the four are joined.
template <int DT, bool TOP>
__global__ void __launch_bounds__(kBlock) logprob_join(const Logprobs q) {
    __shared__ Sums part[kBlock / kWave];
    __shared__ Best lists[kBlock / kWave][kMaxTop];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const float c = q.scale * kLog2e;
    for (int64_t r = blockIdx.x; r < q.rows; r += gridDim.x) {
        const Sums* sums = q.part_sums + r * q.pieces;
        Sums t = {kLowest, 0.0f, 0.0f};
        for (int i = wave * kWave + lane; i < q.pieces; i += kBlock) t = joined(t, sums[i], c);
        const float m = max64(t.m);
        rebase(t, m, c);
        t.s = sum64(t.s);
        t.a = sum64(t.a);
        Best best = {-INFINITY, 0xFFFFFFFFu};
        if constexpr (TOP) {
            const Best* list = q.part_best + r * q.pieces * q.top;
            const int n = q.pieces * q.top;
            for (int i0 = wave * kWave; i0 < n; i0 += kBlock) {
                Best mine = {-INFINITY, 0xFFFFFFFFu};
                if (i0 + lane < n) mine = list[i0 + lane];
                if (__ballot(better(mine.x, mine.j, lane_value(best.x, q.top - 1), lane_word(best.j, q.top - 1)))) merge_unsorted(best, mine);
            }
        }
        join_waves<TOP>(t, best, c, part, lists);
        if (wave == 0) finish<DT>(q, r, t, best);
    }
}

struct LogprobsGrad {
    const void *logits, *tokens;
    const float *stats, *entropy, *g_logp, *g_entropy;
    void* dlogits;
    int64_t ld, ld_out, rows;
    int V, token_bits, chunks;
    float scale;
    bool stream;
};

// 1 - e^u for u <= 0: near 0 its series (the first term left out is below 2^-25 of it), else a difference that loses nothing.
__device__ __forceinline__ float one_less_exp(float u) {
    float s = 1.0f;
#pragma unroll
    for (int k = 8; k >= 2; --k) s = fmaf(u * (1.0f / k), s, 1.0f);
    return u < -0.5f ? 1.0f - exp2_hw(u * kLog2e) : -u * s;
}

// T threads on a chunk of a row, VECS vectors each.  The gradient is p (A + B log2 p) with A and B the row's, and
// log2 p = c (x - m) - log2(sum) a difference and a fused operation; what rounding log2(sum) cut off is in A and B.  Counted:
// 9.6 vector instructions an element, 11.8 with the entropy.
template <int DT, int T, int VECS, bool ENTROPY, Caching BOTH>
__global__ void __launch_bounds__(kBlock) logprob_grad(const LogprobsGrad q) {
    using V = RowVec<DT>;
    constexpr int N = V::kN, R = kBlock / T;
    constexpr int64_t kSize = sizeof(typename V::Elem);
    const int t = threadIdx.x % T;
    const float c = q.scale * kLog2e;
    const int64_t items = q.rows * q.chunks;
    for (int64_t item = (int64_t)blockIdx.x * R + (R > 1 ? threadIdx.x / T : 0); item < items; item += (int64_t)gridDim.x * R) {
        const int64_t r = q.chunks == 1 ? item : item / q.chunks;
        const int64_t first = (item - r * q.chunks) * (T * VECS * N);
        const char* row = static_cast<const char*>(q.logits) + (r * q.ld + first) * kSize;
        char* out = static_cast<char*>(q.dlogits) + (r * q.ld_out + first) * kSize;
        const int left = (int)(q.V - first);
        V x[VECS];
#pragma unroll
        for (int v = 0; v < VECS; ++v) x[v] = load_row<DT, BOTH>(row, (v * T + t) * N, left);
        const float m = q.stats[2 * r], logs = q.stats[2 * r + 1];
        int64_t token = -1;
        float g = 0.0f, h = 0.0f, H = 0.0f;
        if (q.g_logp) {
            token = q.token_bits == 64 ? static_cast<const int64_t*>(q.tokens)[r] : (int64_t) static_cast<const int32_t*>(q.tokens)[r];
            g = token >= q.V ? NAN : token >= 0 ? q.g_logp[r] * q.scale : 0.0f;
        }
        if constexpr (ENTROPY) {
            h = q.g_entropy[r] * q.scale;
            H = q.entropy[r];
        }
        const bool empty = logs == -INFINITY;
        const float l2 = mul_rn(empty ? 0.0f : logs, kLog2e), off = empty ? 0.0f : fmaf(logs, kLog2e, -l2), back = exp2_hw(-off);
        if (empty) g = token >= q.V ? NAN : 0.0f, h = 0.0f;
        const float B = -h * kLn2 * back, A = -(g + h * (H - kLn2 * off)) * back;
        // the token's place in this chunk; one outside the vocabulary has none
        const int at = token >= first && token < q.V && token - first < T * VECS * N ? (int)(token - first) : -1;
#pragma unroll
        for (int v = 0; v < VECS; ++v) {
            const int e = (v * T + t) * N;
            float d[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float l = fmaf(x[v].get(i) - m, c, -l2), p = exp2_hw(l);
                d[i] = ENTROPY ? p * fmaf(B, fmaxf(l, kFloor2), A) : p * A;
            }
            if (at >= e && at < e + N) {
                // g (1 - p) from ln p: 1 - p of a token that is almost certain would be what p's rounding left of it (16384 x 100
                // fp32 8.4 us as that difference, 9.1 so; 8192 x 65536 bf16 357 and 361)
                float y = 0.0f;
#pragma unroll
                for (int i = 0; i < N; ++i) y = e + i == at ? x[v].get(i) - m : y;
                float own = g * one_less_exp(y * q.scale - (empty ? 0.0f : logs));
                if constexpr (ENTROPY) {
                    const float l = fmaf(y, c, -l2);
                    own += exp2_hw(l) * fmaf(B, fmaxf(l, kFloor2), -(h * (H - kLn2 * off)) * back);
                }
#pragma unroll
                for (int i = 0; i < N; ++i) d[i] = e + i == at ? own : d[i];
            }
            V o;
            o.set(d);
            store_row<DT, BOTH>(out, e, left, o);
        }
    }
}

unsigned grid_of(int64_t items) { return (unsigned)(items < (1 << 20) ? items : (1 << 20)); }

// How rows are cut.  A workgroup looks through 2 * 256 vectors at once, so a piece is at least one such chunk; rows that
// are fewer than the workgroups the chip holds are cut until there are about 1024 pieces.  bf16, in pieces and whole: 4 x 131072 5.7
// and 13.9 us, 128 x 131072 12.3 and 15.4, 256 x 131072 19.5 and 24.4; near the rule's end the second kernel costs more than the
// pieces bring, 256 x 50021 11.1 and 10.0, 511 x 131072 31.6 and 29.0.  Rows of one chunk are many from 1024 on: a wavefront each
// and a workgroup each 3.7 and 4.7 us at 1024 x 1000, 5.7 and 5.5 at 1024 x 4000, 8.5 and 16.6 at 8192 x 1000, but 4.8 and
// 3.9 at 256 x 4000, and 12.6 and 9.3 there with five alternatives.
struct Cut {
    int threads, pieces, piece;
};

Cut cut_rows(int64_t rows, int64_t V, int dt) {
    const int64_t chunk = (dt == SDGP_BF16 ? 8 : 4) * kAtOnce * (int64_t)kBlock;
    if (V <= chunk) return {rows >= 1024 ? kWave : kBlock, 1, (int)V};
    int64_t pieces = rows >= 512 ? 1 : 1024 / rows;
    const int64_t most = (V + chunk - 1) / chunk;
    pieces = pieces > most ? most : pieces;
    const int64_t piece = ((V + pieces - 1) / pieces + chunk - 1) / chunk * chunk;
    return {kBlock, (int)((V + piece - 1) / piece), (int)(piece < V ? piece : V)};
}

template <int DT, bool TOP>
int launch_rows(const Logprobs& q, const Cut& cut, hipStream_t stream) {
    const int64_t items = q.rows * cut.pieces;
    if (cut.threads == kWave)
        hipLaunchKernelGGL((logprob_rows<DT, kWave, TOP, kKeep>), dim3(grid_of((items + 3) / 4)), dim3(kBlock), 0, stream, q);
    else if (q.stream)
        hipLaunchKernelGGL((logprob_rows<DT, kBlock, TOP, kStream>), dim3(grid_of(items)), dim3(kBlock), 0, stream, q);
    else
        hipLaunchKernelGGL((logprob_rows<DT, kBlock, TOP, kKeep>), dim3(grid_of(items)), dim3(kBlock), 0, stream, q);
    const int rc = launch_status();
    if (rc != SDGP_OK || cut.pieces == 1) return rc;
    hipLaunchKernelGGL((logprob_join<DT, TOP>), dim3(grid_of(q.rows)), dim3(kBlock), 0, stream, q);
    return launch_status();
}

template <int DT, bool ENTROPY>
int launch_grad(LogprobsGrad q, hipStream_t stream) {
    constexpr int N = RowVec<DT>::kN;
    const auto go = [&](auto kernel, int threads, int vecs) {
        q.chunks = (int)((q.V + threads * vecs * N - 1) / (threads * vecs * N));
        const int64_t items = q.rows * q.chunks, at_once = kBlock / threads;
        hipLaunchKernelGGL(kernel, dim3(grid_of((items + at_once - 1) / at_once)), dim3(kBlock), 0, stream, q);
        return launch_status();
    };
    const auto sized = [&](auto both) {
        constexpr Caching C = decltype(both)::value;
        if (q.V <= 16 * N) return go(logprob_grad<DT, 16, 1, ENTROPY, C>, 16, 1);
        if (q.V <= 64 * 2 * N) return go(logprob_grad<DT, 64, 2, ENTROPY, C>, 64, 2);
        if (q.V <= 256 * 8 * N) return go(logprob_grad<DT, 256, 2, ENTROPY, C>, 256, 2);
        return go(logprob_grad<DT, 256, 4, ENTROPY, C>, 256, 4);
    };
    return q.stream ? sized(Cached<kStream>{}) : sized(Cached<kKeep>{});
}

}  // namespace

// Logits that a 256 MB cache keeps nothing of for the gradient are read with the streaming hint, where rows begin on 16 bytes
// (forward of 8192 x 65536 bf16 182 us without, 167 with it); and from 80 MB on logits and gradients pass by the caches in
// the backward kernel.  By itself that kernel is always quicker so (bf16 x 32768, kept and past: 16 MB 9.7 and 7.5 us, 84 MB
// 36.2 and 32.4, 268 MB 99 and 94); but what is kept is there for the layer that reads the gradient next (forward, gradient and a pruned
// layer of 256 inputs: 67 MB 210 and 240 us, 84 MB 218 and 249, 134 MB 265 and 279, 268 MB 364 and 354).
static bool larger_than(int64_t megabytes, int64_t rows, int64_t V, int dt) { return rows * V * (dt == SDGP_BF16 ? 2 : 4) > megabytes << 20; }

size_t token_logprobs_workspace(int64_t rows, int64_t V, int dt, int top) {
    if (rows == 0) return 0;
    const Cut cut = cut_rows(rows, V, dt);
    return cut.pieces == 1 ? 0 : (size_t)rows * cut.pieces * (sizeof(Sums) + top * sizeof(Best));
}

int token_logprobs_launch(const void* logits, int64_t ld, const void* tokens, int token_bits, float* logp, float* entropy,
                          float* top_logp, int64_t* top_ids, float* stats, int64_t rows, int64_t V, int dt, int top, float scale,
                          void* workspace, hipStream_t stream) {
    const Cut cut = cut_rows(rows, V, dt);
    const int64_t items = rows * cut.pieces;
    Best* lists = static_cast<Best*>(workspace);
    const Logprobs q = {logits, tokens, logp, entropy, top_logp, stats, top_ids, ld, rows, (int)V, top, token_bits, scale, cut.pieces,
                        cut.piece, reinterpret_cast<Sums*>(lists + items * top), lists,
                        larger_than(256, rows, V, dt) && is_aligned16(logits) && ld * (dt == SDGP_BF16 ? 2 : 4) % 16 == 0};
    if (dt == SDGP_BF16) return top > 0 ? launch_rows<SDGP_BF16, true>(q, cut, stream) : launch_rows<SDGP_BF16, false>(q, cut, stream);
    return top > 0 ? launch_rows<SDGP_F32, true>(q, cut, stream) : launch_rows<SDGP_F32, false>(q, cut, stream);
}

int token_logprobs_bwd_launch(const void* logits, int64_t ld, const void* tokens, int token_bits, const float* stats, const float* entropy,
                              const float* g_logp, const float* g_entropy, void* dlogits, int64_t ld_out, int64_t rows, int64_t V,
                              int dt, float scale, hipStream_t stream) {
    const LogprobsGrad q = {logits, tokens, stats, entropy, g_logp, g_entropy, dlogits, ld, ld_out, rows, (int)V, token_bits, 1, scale,
                            larger_than(80, rows, V, dt)};
    if (dt == SDGP_BF16) return g_entropy ? launch_grad<SDGP_BF16, true>(q, stream) : launch_grad<SDGP_BF16, false>(q, stream);
    return g_entropy ? launch_grad<SDGP_F32, true>(q, stream) : launch_grad<SDGP_F32, false>(q, stream);
}

}  // namespace sdgp
