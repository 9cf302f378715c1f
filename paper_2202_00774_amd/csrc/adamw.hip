// One AdamW step over many tensors.
//
//   g = grad * grad_scale;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
//   p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// States in 8 bits hold m and r = sqrt(v) as e4m3 codes with one scale, a power of two, for each 256 elements: the
// smallest code is 2^-9 where a block's largest value is between 224 and 448, so codes reach down to 2^-17 of it, and with the
// root stored that is 2^-17 of the largest step size too.
// Both are rounded up or down at random, with the probability of what is cut off: v moves by a thousandth a step, far
// less than half the distance of two codes, so rounded to the nearest it would never move again.  The random word is
// the library's counter hash of (seed, element), so a step can be repeated bit for bit.  A root that is not zero is not
// stored as zero, since the step divides by it.  A gradient that is infinite or NaN spoils its own element only: the
// scale is taken over the block's finite values.
//
// Bound by memory: 28 bytes an element with fp32 states (parameter and both states in and out, gradient in), 16 with 8-bit
// ones.  A wavefront takes a block of 256 elements, four a lane, so a block's scale is a maximum over one wavefront.  A
// workgroup's tile of blocks lies in one tensor, which it looks up in the arguments.  In 8 bits an element costs 91 vector
// instructions, ten of them the step's division: codes are cut from the float's bits, and what only infinities and NaN
// need is done where a block has them.  Measured: 24 x 8388608 elements with bf16 gradients in 8 bits 562 us (5.8 TB/s; the vector
// pipes are busy for 94 % of them), in fp32 1010 (6.0 TB/s); ResNet-50's 161 tensors 91 and 135.
#include "adamw.h"

#include "rows.h"

namespace sdgp {

namespace {

constexpr int kThreads = 256, kWave = 64;
constexpr uint32_t kInf = 0x7F800000u;

// One mixed word of (seed, element): the finalizer of common.h's hash, one word an element.
__device__ __forceinline__ uint32_t random_word(uint32_t row, uint32_t e) {
    uint32_t v = row ^ e;
    v ^= v >> 16;
    v *= 0x6A09E667u;
    v ^= v >> 15;
    v *= 0xBB67AE85u;
    return v ^ (v >> 16);
}

// Largest over the wavefront: of the bits of floats that are not negative, which are in the floats' order.
__device__ __forceinline__ uint32_t max_bits(uint32_t v) {
    const auto dpp = [](uint32_t x, auto ctrl) {
        return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xF, 0xF, true);
    };
    v = max(v, dpp(v, std::integral_constant<int, 0xB1>{}));
    v = max(v, dpp(v, std::integral_constant<int, 0x4E>{}));
    v = max(v, dpp(v, std::integral_constant<int, 0x141>{}));
    v = max(v, dpp(v, std::integral_constant<int, 0x140>{}));
    const auto lane = [&](int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); };
    return max(max(lane(0), lane(16)), max(lane(32), lane(48)));
}

// The exponent k of a block's scale 2^k, from the bits of its largest value: the smallest with top <= 448 * 2^k, -126 at
// least; 0 for a block of zeros.  448 is 1.75 * 2^8, so k is the exponent less 8, one more above 1.75 (subnormal tops end up
// at -126 either way).
__device__ __forceinline__ int scale_exponent(uint32_t top) {
    if (top == 0) return 0;
    const int k = (int)(top >> 23) - 127 - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return k < -126 ? -126 : k;
}

__device__ __forceinline__ float power_of_two(int k) { return bits_to_float((uint32_t)(k + 127) << 23); }

// |x| / 2^k, at most 448, on the grid of e4m3, rounded up where u / 2^16 exceeds what is cut off.  Another 120 off the
// exponent, a float's exponent and upper three mantissa bits are the code, subnormal codes being where a float's subnormals
// are; u is added below them.  (What lies under 2^-6 is rounded to 2^-20 of a code's step by that.)
__device__ __forceinline__ uint32_t to_code(float x, int k, uint32_t u) {
    return (float_to_bits(ldexpf(fabsf(x), -k - 120)) + (u << 4)) >> 20;
}

typedef uint32_t u32x2_half_aligned __attribute__((ext_vector_type(2), aligned(2), may_alias));
typedef uint32_t u32_any __attribute__((aligned(1), may_alias));

// Four values of a lane: elements e .. e + 3 of a tensor of n.  What lies outside is 0 and is neither read nor written.
// Everything passes by once a step, so loads and stores have the streaming hint (582 us without, 562 with it, for 24 x 8388608
// elements in 8 bits; 1112 and 1011 in fp32; 156 and 136 for ResNet-50's tensors in fp32).
template <int DT>
__device__ __forceinline__ void load4(const void* p, int64_t e, int64_t n, float (&f)[4]) {
    if (e + 4 <= n) {
        if constexpr (DT == SDGP_BF16) {
            const auto v = __builtin_nontemporal_load(reinterpret_cast<const u32x2_half_aligned*>(static_cast<const uint16_t*>(p) + e));
#pragma unroll
            for (int i = 0; i < 2; ++i) f[2 * i] = bits_to_float(v[i] << 16), f[2 * i + 1] = bits_to_float(v[i] & 0xFFFF0000u);
        } else {
            const auto v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_word_aligned*>(static_cast<const float*>(p) + e));
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = bits_to_float(v[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[i] = 0.0f;
            if (e + i < n) f[i] = DT == SDGP_BF16 ? bf16_to_float(static_cast<const uint16_t*>(p)[e + i]) : static_cast<const float*>(p)[e + i];
        }
    }
}

template <int DT>
__device__ __forceinline__ void store4(void* p, int64_t e, int64_t n, const float (&f)[4]) {
    if (e + 4 <= n) {
        if constexpr (DT == SDGP_BF16) {
            const u32x2_half_aligned v = {float2_to_bf16x2(f[0], f[1]), float2_to_bf16x2(f[2], f[3])};
            __builtin_nontemporal_store(v, reinterpret_cast<u32x2_half_aligned*>(static_cast<uint16_t*>(p) + e));
        } else {
            const u32x4_word_aligned v = {float_to_bits(f[0]), float_to_bits(f[1]), float_to_bits(f[2]), float_to_bits(f[3])};
            __builtin_nontemporal_store(v, reinterpret_cast<u32x4_word_aligned*>(static_cast<float*>(p) + e));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (e + i < n) {
                if constexpr (DT == SDGP_BF16) static_cast<uint16_t*>(p)[e + i] = (uint16_t)float2_to_bf16x2(f[i], 0.0f);
                else static_cast<float*>(p)[e + i] = f[i];
            }
    }
}

__device__ __forceinline__ uint32_t load4_codes(const void* p, int64_t e, int64_t n) {
    const uint8_t* at = static_cast<const uint8_t*>(p) + e;
    if (e + 4 <= n) return __builtin_nontemporal_load(reinterpret_cast<const u32_any*>(at));
    uint32_t v = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (e + i < n) v |= (uint32_t)at[i] << (8 * i);
    return v;
}

__device__ __forceinline__ void store4_codes(void* p, int64_t e, int64_t n, uint32_t v) {
    uint8_t* at = static_cast<uint8_t*>(p) + e;
    if (e + 4 <= n) {
        __builtin_nontemporal_store(v, reinterpret_cast<u32_any*>(at));
        return;
    }
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (e + i < n) at[i] = (uint8_t)(v >> (8 * i));
}

__device__ __forceinline__ void from_codes(uint32_t v, float scale, float (&f)[4]) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)v, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)v, true);
    f[0] = lo[0] * scale, f[1] = lo[1] * scale, f[2] = hi[0] * scale, f[3] = hi[1] * scale;
}

// The codes of a block's four values a lane; KEEP: not negative, and what is not zero is not stored as zero.
template <bool KEEP>
__device__ __forceinline__ uint32_t to_codes(float (&x)[4], const uint32_t (&u)[4], float* scale_at) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) most = max(most, float_to_bits(x[i]) & 0x7FFFFFFFu);
    uint32_t top = max_bits(most);
    const bool odd = top >= kInf;       // something infinite or NaN: the scale is that of the others
    uint32_t spoilt = 0;                // the code of NaN in their places
    if (odd) {
        most = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t b = float_to_bits(x[i]) & 0x7FFFFFFFu;
            if (b >= kInf) x[i] = 0.0f, spoilt |= 0x7Fu << (8 * i);
            else most = max(most, b);
        }
        top = max_bits(most);
    }
    const int k = scale_exponent(top);
    if ((threadIdx.x & (kWave - 1)) == 0) *scale_at = power_of_two(k);
    uint32_t codes = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t b = float_to_bits(x[i]);
        uint32_t code = to_code(x[i], k, u[i]);
        if constexpr (KEEP) code = max(code, min(b, 1u));
        else code |= (b >> 24) & 0x80u;
        codes |= code << (8 * i);
    }
    return codes | spoilt;   // a 0, whatever its random bits, is stored as 0
}

template <int PDT, int GDT, int BITS>
__global__ void __launch_bounds__(kThreads) adamw_tiles(const AdamArgs<BITS> a) {
    using Tensors = AdamTensors<BITS>;
    constexpr int kTile = adam_tile(BITS), kAtOnce = kTile / (kThreads / kWave);   // blocks of a wavefront
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    // the last tensor that begins at this tile or before it; every lane compares one or two (a search would wait for each step)
    int at = -1;
#pragma unroll
    for (int i = 0; i < Tensors::kMost; i += kWave) {
        const int mine = i + lane < Tensors::kMost ? i + lane : Tensors::kMost - 1;
        at += __builtin_popcountll(__ballot(i + lane < a.count && a.t.first[mine] <= blockIdx.x));
    }
    struct {
        void* p;
        const void* g;
        void *m, *v;
        uint16_t* copy;
    } const t = {a.t.p[at], a.t.g[at], a.t.m[at], a.t.v[at], a.t.copy[at]};
    const int64_t block0 = (int64_t)(blockIdx.x - a.t.first[at]) * kTile + wave * kAtOnce, n = a.t.n[at];
    if (block0 * kAdamBlock >= n) return;
    float *m_scale = nullptr, *v_scale = nullptr;
    if constexpr (BITS == 8) m_scale = a.t.m_scale[at], v_scale = a.t.v_scale[at];
    const float gs = a.grad_scale ? *a.grad_scale : 1.0f;

    float p[kAtOnce][4], g[kAtOnce][4], m[kAtOnce][4], v[kAtOnce][4];
    uint32_t mc[kAtOnce], vc[kAtOnce];
#pragma unroll
    for (int b = 0; b < kAtOnce; ++b) {
        const int64_t e = (block0 + b) * kAdamBlock + lane * 4;
        load4<PDT>(t.p, e, n, p[b]);
        load4<GDT>(t.g, e, n, g[b]);
        if constexpr (BITS == 32) {
            load4<SDGP_F32>(t.m, e, n, m[b]);
            load4<SDGP_F32>(t.v, e, n, v[b]);
        } else {
            mc[b] = load4_codes(t.m, e, n);
            vc[b] = load4_codes(t.v, e, n);
        }
    }
#pragma unroll
    for (int b = 0; b < kAtOnce; ++b) {
        const int64_t block = block0 + b, e = block * kAdamBlock + lane * 4;
        if (block * kAdamBlock >= n) break;
        if constexpr (BITS == 8) {
            from_codes(mc[b], m_scale[block], m[b]);
            from_codes(vc[b], v_scale[block], v[b]);
        }
        float r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // one rounding an operation, so that a code does not depend on which products were fused
            const float gi = mul_rn(g[b][i], gs), v0 = BITS == 8 ? mul_rn(v[b][i], v[b][i]) : v[b][i];
            m[b][i] = add_rn(mul_rn(m[b][i], a.b1), mul_rn(gi, a.one_b1));
            v[b][i] = add_rn(mul_rn(v0, a.b2), mul_rn(mul_rn(gi, gi), a.one_b2));
            r[i] = sqrtf(v[b][i]);
            const float den = fmaf(r[i], a.inv_root_bc2, a.eps);
            p[b][i] = fmaf(p[b][i], a.decay, -a.rate * (m[b][i] / den));
        }
        store4<PDT>(t.p, e, n, p[b]);
        if (PDT == SDGP_F32 && t.copy != nullptr) store4<SDGP_BF16>(t.copy, e, n, p[b]);
        if constexpr (BITS == 32) {
            store4<SDGP_F32>(t.m, e, n, m[b]);
            store4<SDGP_F32>(t.v, e, n, v[b]);
        } else {
            const uint64_t from = ((uint64_t)a.t.block[at] + block) * kAdamBlock;
            const uint32_t row = hash_row(a.mix, (uint32_t)(from >> 32)), e32 = (uint32_t)from + lane * 4;
            uint32_t um[4], uv[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t w = random_word(row, e32 + i);
                um[i] = w & 0xFFFFu, uv[i] = w >> 16;
            }
            store4_codes(t.m, e, n, to_codes<false>(m[b], um, m_scale + block));
            store4_codes(t.v, e, n, to_codes<true>(r, uv, v_scale + block));
        }
    }
}

}  // namespace

template <int BITS>
int adamw_launch(const AdamArgs<BITS>& a, uint32_t tiles, int param_dt, int grad_dt, hipStream_t stream) {
    const bool pb = param_dt == SDGP_BF16, gb = grad_dt == SDGP_BF16;
    auto k = pb ? (gb ? adamw_tiles<SDGP_BF16, SDGP_BF16, BITS> : adamw_tiles<SDGP_BF16, SDGP_F32, BITS>)
                : (gb ? adamw_tiles<SDGP_F32, SDGP_BF16, BITS> : adamw_tiles<SDGP_F32, SDGP_F32, BITS>);
    hipLaunchKernelGGL(k, dim3(tiles), dim3(kThreads), 0, stream, a);
    return launch_status();
}

template int adamw_launch<8>(const AdamArgs<8>& a, uint32_t tiles, int param_dt, int grad_dt, hipStream_t stream);
template int adamw_launch<32>(const AdamArgs<32>& a, uint32_t tiles, int param_dt, int grad_dt, hipStream_t stream);

}  // namespace sdgp
