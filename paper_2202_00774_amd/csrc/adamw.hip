// One AdamW step over many tensors.
//
//   g = grad * grad_scale;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
//   p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// States in 8 bits hold m and r = sqrt(v) as e4m3 codes with one scale, a power of two, for each 256 elements: codes
// reach down to 2^-18 of a block's largest value, and with the root stored that is 2^-18 of the largest step size too.
// Both are rounded up or down at random, with the probability of what is cut off: v moves by a thousandth a step, far
// less than half the distance of two codes, so rounded to the nearest it would never move again.  The random word is
// the library's counter hash of (seed, element), so a step can be repeated bit for bit.  A root that is not zero is not
// stored as zero, since the step divides by it.  A gradient that is infinite or NaN spoils its own element only: the
// scale is taken over the block's finite values.
#include "adamw.h"

namespace sdgp {

namespace {

constexpr float kMaxFinite = 3.402823466e38f;

// One mixed word of (seed, element): the finalizer of common.h's hash, one word an element.
__device__ __forceinline__ uint32_t random_word(uint32_t mix, uint64_t e) {
    uint32_t v = hash_row(mix, (uint32_t)(e >> 32)) ^ (uint32_t)e;
    v ^= v >> 16;
    v *= 0x6A09E667u;
    v ^= v >> 15;
    v *= 0xBB67AE85u;
    return v ^ (v >> 16);
}

// Largest over the 256 threads of the workgroup.
__device__ __forceinline__ float block_max(float v, float* lds) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v = fmaxf(v, __shfl_xor(v, o));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    return fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
}

// The exponent k of a block's scale 2^k: the smallest with top <= 448 * 2^k, -126 at least; 0 for a block of zeros.
__device__ __forceinline__ int scale_exponent(float top) {
    if (!(top > 0.0f)) return 0;
    int e;
    const float f = frexpf(top, &e);
    const int k = e - 9 + (f > 0.875f ? 1 : 0);
    return k < -126 ? -126 : k;
}

__device__ __forceinline__ float power_of_two(int k) { return bits_to_float((uint32_t)(k + 127) << 23); }

// x / 2^k on the grid of e4m3 (8 steps a power of two, evenly spaced below 2^-6), rounded up where u exceeds what is
// cut off; the code's eight bits.
__device__ __forceinline__ uint32_t to_code(float x, int k, float u, bool keep) {
    if (!(fabsf(x) <= kMaxFinite)) return 0x7Fu;
    const float y = ldexpf(fabsf(x), -k);
    int e = (int)(float_to_bits(y) >> 23) - 127;
    e = e < -6 ? -6 : e;
    float c = floorf(ldexpf(y, 3 - e) + u);
    if (keep && y > 0.0f && c == 0.0f) c = 1.0f;
    const uint32_t sign = (float_to_bits(x) >> 24) & 0x80u;
    // c in 0 .. 16 steps of 2^(e-3): a step past 15 is the next power of two's first code
    return sign | ((uint32_t)((e + 6) << 3) + (uint32_t)c);
}

__device__ __forceinline__ float from_code(uint32_t code) {
    const uint32_t e = (code >> 3) & 15u, f = code & 7u;
    const float v = e ? ldexpf((float)(8u + f), (int)e - 10) : ldexpf((float)f, -9);
    return (code & 0x7Fu) == 0x7Fu ? NAN : (code & 0x80u) ? -v : v;
}

template <int PDT, int GDT, int BITS>
__global__ void __launch_bounds__(kAdamBlock) adamw_blocks(const AdamArgs a) {
    __shared__ float lds[4];
    int lo = 0, hi = a.count;                       // the tensor that holds this block
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.first[mid] <= blockIdx.x) lo = mid;
        else hi = mid;
    }
    const AdamTensor& t = a.t[lo];
    const int64_t block = blockIdx.x - a.first[lo], i = block * kAdamBlock + threadIdx.x;
    const bool in = i < t.n;
    const float gs = a.grad_scale ? *a.grad_scale : 1.0f;

    float p = 0.0f, g = 0.0f, m = 0.0f, v = 0.0f;
    if (in) {
        p = PDT == SDGP_BF16 ? bf16_to_float(static_cast<uint16_t*>(t.p)[i]) : static_cast<float*>(t.p)[i];
        g = GDT == SDGP_BF16 ? bf16_to_float(static_cast<const uint16_t*>(t.g)[i]) : static_cast<const float*>(t.g)[i];
        if constexpr (BITS == 32) {
            m = static_cast<float*>(t.m)[i];
            v = static_cast<float*>(t.v)[i];
        } else {
            m = from_code(static_cast<uint8_t*>(t.m)[i]) * t.m_scale[block];
            const float r = from_code(static_cast<uint8_t*>(t.v)[i]) * t.v_scale[block];
            v = __fmul_rn(r, r);
        }
    }
    // one rounding an operation, so that a code does not depend on which products were fused
    g = __fmul_rn(g, gs);
    m = __fadd_rn(__fmul_rn(m, a.b1), __fmul_rn(g, a.one_b1));
    v = __fadd_rn(__fmul_rn(v, a.b2), __fmul_rn(__fmul_rn(g, g), a.one_b2));
    const float r = sqrtf(v);
    p = p * a.decay - a.rate * (m / (r / a.root_bc2 + a.eps));
    if (in) {
        if constexpr (PDT == SDGP_BF16) static_cast<uint16_t*>(t.p)[i] = (uint16_t)float_to_bf16(p);
        else static_cast<float*>(t.p)[i] = p;
        if (t.copy) t.copy[i] = (uint16_t)float_to_bf16(p);
    }
    if constexpr (BITS == 32) {
        if (in) {
            static_cast<float*>(t.m)[i] = m;
            static_cast<float*>(t.v)[i] = v;
        }
    } else {
        const float am = fabsf(m);
        const int km = scale_exponent(block_max(am <= kMaxFinite ? am : 0.0f, lds));
        const int kv = scale_exponent(block_max(r <= kMaxFinite ? r : 0.0f, lds));
        if (in) {
            const uint32_t w = random_word(a.mix, ((uint64_t)a.base + blockIdx.x) * kAdamBlock + threadIdx.x);
            static_cast<uint8_t*>(t.m)[i] = (uint8_t)to_code(m, km, (float)(w & 0xFFFFu) * 0x1p-16f, false);
            static_cast<uint8_t*>(t.v)[i] = (uint8_t)to_code(r, kv, (float)(w >> 16) * 0x1p-16f, true);
        }
        if (threadIdx.x == 0) {
            t.m_scale[block] = power_of_two(km);
            t.v_scale[block] = power_of_two(kv);
        }
    }
}

}  // namespace

int adamw_launch(const AdamArgs& a, int param_dt, int grad_dt, int state_bits, hipStream_t stream) {
    const dim3 grid(a.first[a.count]), block(kAdamBlock);
    const bool pb = param_dt == SDGP_BF16, gb = grad_dt == SDGP_BF16;
    if (state_bits == 32) {
        auto k = pb ? (gb ? adamw_blocks<SDGP_BF16, SDGP_BF16, 32> : adamw_blocks<SDGP_BF16, SDGP_F32, 32>)
                    : (gb ? adamw_blocks<SDGP_F32, SDGP_BF16, 32> : adamw_blocks<SDGP_F32, SDGP_F32, 32>);
        hipLaunchKernelGGL(k, grid, block, 0, stream, a);
    } else {
        auto k = pb ? (gb ? adamw_blocks<SDGP_BF16, SDGP_BF16, 8> : adamw_blocks<SDGP_BF16, SDGP_F32, 8>)
                    : (gb ? adamw_blocks<SDGP_F32, SDGP_BF16, 8> : adamw_blocks<SDGP_F32, SDGP_F32, 8>);
        hipLaunchKernelGGL(k, grid, block, 0, stream, a);
    }
    return launch_status();
}

}  // namespace sdgp
