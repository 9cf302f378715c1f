// Rotary positions: pairs of a head's values turned by angles that are position times frequency.
//
//   (a, b) -> (a cos - b sin, a sin + b cos),  angle of pair i = position[axis of i] * freqs[i];  inverse: sin with the other sign
// Bound by memory: queries and keys are read and written once.  A workgroup computes its tokens' sines and cosines first, one a
// thread, and keeps them in LDS for all heads.  Angles are counted in turns in twice 64 bits, so positions up to 2^53 lose nothing;
// of what is left after whole turns, at most half a one, 32 bits are enough.
#include "fastdiv.h"
#include "rotary.h"
#include "rows.h"

namespace sdgp {

namespace {

constexpr int kBlock = 256;

// position * frequency / 2 pi as a sum of two numbers, less the whole turns of the first: exact products and their errors, so
// none of them may be fused with what follows it.
__device__ __forceinline__ float part_of_a_turn(double position, double freq) {
#pragma clang fp contract(off)
    constexpr double kTurn = 0.15915494309189535, kTurnLow = -9.839338337591243e-18;
    const double angle = position * freq, angle_low = fma(position, freq, -angle);
    const double turns = angle * kTurn, low = fma(angle, kTurn, -turns) + (angle * kTurnLow + angle_low * kTurn);
    return (float)((turns - rint(turns)) + low);
}

template <int DT, bool INTERLEAVED>
__global__ void __launch_bounds__(kBlock) rotary_kernel(const Rotary a) {
    constexpr int N = RowVec<DT>::kN, SIZE = 16 / N;
    extern __shared__ float lds[];                      // [tokens, 2, F]: cosines, sines
    const int F = a.F;
    const int64_t first = (int64_t)blockIdx.x * a.tokens;
    const int tokens = (int)(a.T - first < a.tokens ? a.T - first : a.tokens);
    for (int e = threadIdx.x; e < tokens * F; e += kBlock) {
        const int j = (int)divide((uint32_t)e, a.by_pairs), i = e - j * F;
        int axis = 0;
        while (axis + 1 < a.axes && i >= a.end[axis]) ++axis;
        const int64_t at = (first + j) * a.axes + axis;
        const double position = a.position_bits == 64 ? (double)static_cast<const int64_t*>(a.positions)[at]
                                                      : (double)static_cast<const int32_t*>(a.positions)[at];
        float s, c;
        sincospif(2.0f * part_of_a_turn(position, (double)a.freqs[i]), &s, &c);
        lds[(2 * j) * F + i] = c;
        lds[(2 * j + 1) * F + i] = a.inverse ? -s : s;
    }
    __syncthreads();
    const int all = tokens * a.per_token;               // per_token: chunks of all heads
    for (int e = threadIdx.x; e < all; e += kBlock) {
        const int j = (int)divide((uint32_t)e, a.by_token), r = e - j * a.per_token;
        const int h = (int)divide((uint32_t)r, a.by_head), chunk = r - h * a.per_head;
        const bool key = h >= a.H;
        const int64_t t = first + j;
        const char* in = key ? static_cast<const char*>(a.k) + (t * a.k_token + (h - a.H) * a.k_head) * SIZE
                             : static_cast<const char*>(a.q) + (t * a.q_token + h * a.q_head) * SIZE;
        char* out = key ? static_cast<char*>(a.k_out) + (t * a.k_out_token + (h - a.H) * a.k_out_head) * SIZE
                        : static_cast<char*>(a.q_out) + (t * a.q_out_token + h * a.q_out_head) * SIZE;
        const float *cosine = lds + (2 * j) * F, *sine = cosine + F;
        if (chunk >= a.turned) {                        // what is not turned
            if (in == out) continue;
            const int at = (chunk - a.turned) * N;
            store_row<DT>(out + 2 * F * SIZE, at, a.D - 2 * F, load_row<DT>(in + 2 * F * SIZE, at, a.D - 2 * F));
            continue;
        }
        const int at = chunk * N;
        if constexpr (INTERLEAVED) {
            const auto x = load_row<DT>(in, at, 2 * F);
            float y[N];
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                const int p = at / 2 + i / 2 < F ? at / 2 + i / 2 : 0;
                const float c = cosine[p], s = sine[p], u = x.get(i), v = x.get(i + 1);
                y[i] = u * c - v * s;
                y[i + 1] = u * s + v * c;
            }
            RowVec<DT> z;
            z.set(y);
            store_row<DT>(out, at, 2 * F, z);
        } else {
            const auto x = load_row<DT>(in, at, F), w = load_row<DT>(in + F * SIZE, at, F);
            float y[N], z[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int p = at + i < F ? at + i : 0;
                const float c = cosine[p], s = sine[p], u = x.get(i), v = w.get(i);
                y[i] = u * c - v * s;
                z[i] = u * s + v * c;
            }
            RowVec<DT> one, two;
            one.set(y);
            two.set(z);
            store_row<DT>(out, at, F, one);
            store_row<DT>(out + F * SIZE, at, F, two);
        }
    }
}

}  // namespace

int rotary_launch(Rotary a, int dt, bool interleaved, hipStream_t stream) {
    const int N = dt == SDGP_BF16 ? 8 : 4;
    a.turned = interleaved ? (2 * a.F + N - 1) / N : (a.F + N - 1) / N;
    a.per_head = a.turned + (a.D - 2 * a.F + N - 1) / N;
    a.per_token = a.per_head * (a.H + a.Hk);
    a.by_pairs = fast_div((uint32_t)a.F), a.by_head = fast_div((uint32_t)a.per_head), a.by_token = fast_div((uint32_t)a.per_token);
    a.tokens = rotary_tokens(a.F);
    if (a.tokens > a.T) a.tokens = (int)a.T;
    const dim3 grid((unsigned)((a.T + a.tokens - 1) / a.tokens)), block(kBlock);
    const size_t lds = (size_t)a.tokens * 2 * a.F * sizeof(float);
    if (dt == SDGP_BF16) {
        if (interleaved) hipLaunchKernelGGL((rotary_kernel<SDGP_BF16, true>), grid, block, lds, stream, a);
        else hipLaunchKernelGGL((rotary_kernel<SDGP_BF16, false>), grid, block, lds, stream, a);
    } else {
        if (interleaved) hipLaunchKernelGGL((rotary_kernel<SDGP_F32, true>), grid, block, lds, stream, a);
        else hipLaunchKernelGGL((rotary_kernel<SDGP_F32, false>), grid, block, lds, stream, a);
    }
    return launch_status();
}

}  // namespace sdgp
