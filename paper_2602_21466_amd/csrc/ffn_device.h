// Device helpers of the feed-forward sublayer's kernels: conversions,
// activations and their derivatives, the counter-based generator, and
// reductions over a work-group.  Internal; included by the ffn_*.hip sources.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "ffn_internal.h"

namespace ffn {
namespace dev {

typedef __bf16 bf16;
typedef _Float16 fp16;

template <typename T> __device__ __forceinline__ float to_f32(T v) { return (float)v; }

// act(g) and act'(g).  T: the arrays' type; for 16-bit ones the exponential and the reciprocal are the hardware's (within
// 2^-20 for |g| < 16), and the error function takes the form of Abramowitz and Stegun, 7.1.26, whose exponential is the
// derivative's own: erfc(x) = t (a1 + t (a2 + ...)) exp(-x^2), t = 1 / (1 + p x), x >= 0.  The table's coefficients are for
// the absolute error; those here are fitted to the relative one (least squares, weights after Lawson until the largest
// errors are equal, for x up to 9.5), which decides gelu where the gate has nearly closed: 6.4e-7, and with the 32-bit
// arithmetic 3e-6 for g >= -6 and 4e-5 down to -13.4, below which bf16 has no values: a 150th of fp16's unit roundoff and a
// hundredth of bf16's.  (A 128 x 128 tile's epilogue with erff and expf took as long as 16 steps of its products.)  32-bit
// arrays have the error function beside 1, as the plain form does: its rounding, 2^-24, is what is left of gelu's value there.
template <typename T> __device__ __forceinline__ void activate(int act, float g, float& v, float& dv) {
    constexpr bool kFast = sizeof(T) == 2;
    if (act == FFN_SILU) {
        const float s = kFast ? __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * g)) : 1.0f / (1.0f + expf(-g));
        v = g * s;
        dv = s * (1.0f + g * (1.0f - s));
    } else if (act == FFN_GELU) {
        float c, e;
        if (kFast) {
            e = __builtin_amdgcn_exp2f(-0.72134752f * g * g);       // exp(-g^2 / 2)
            const float t = __builtin_amdgcn_rcpf(1.0f + 0.375f * 0.70710678f * fabsf(g));
            const float half = 0.5f * e * t * (0.21133945f + t * (0.215689163f + t * (0.166664659f + t * (0.283061293f + t * (-0.129596948f + t * (0.387937573f - t * 0.135095828f))))));
            c = g < 0.0f ? half : 1.0f - half;
        } else {
            e = expf(-0.5f * g * g);
            c = 0.5f * (1.0f + erff(g * 0.70710678118654752440f));
        }
        v = g * c;
        dv = c + g * 0.39894228040143267794f * e;
    } else {
        v = g <= 0.0f ? 0.0f : g;   // (NaN stays)
        dv = g > 0.0f ? 1.0f : 0.0f;
    }
}

// Philox 4x32, 10 rounds (Salmon et al. 2011): two 32 x 32 -> 64 bit products a round
// mix the four counter words; the key steps by fixed constants (the golden ratio, sqrt 3 - 1).
struct Words { uint32_t w[4]; };
__device__ __forceinline__ Words philox(uint32_t c0, uint32_t c1, uint64_t offset, uint64_t seed) {
    uint32_t c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p = (uint64_t)0xD2511F53u * c0, q = (uint64_t)0xCD9E8D57u * c2;
        const uint32_t n0 = (uint32_t)(q >> 32) ^ c1 ^ k0, n2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
        c1 = (uint32_t)q;
        c3 = (uint32_t)p;
        c0 = n0;
        c2 = n2;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Words{{c0, c1, c2, c3}};
}

// Whether column (8 b + i) of the block's eight is kept.
__device__ __forceinline__ bool kept(const Words& q, int i, uint32_t threshold) {
    const uint32_t v = q.w[i >> 1];
    return ((i & 1) ? v >> 16 : v & 0xFFFFu) >= threshold;
}

// Sum over the work-group, returned to every thread; `s` holds one float per wave.
__device__ __forceinline__ float group_sum(float v, float* s) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o, 64);
    const int waves = blockDim.x >> 6;
    if (waves == 1) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    float t = s[0];
    for (int i = 1; i < waves; ++i) t += s[i];
    return t;
}

}  // namespace dev
}  // namespace ffn
