// The feed-forward block's forward products for few rows (served tokens): the weights are read once, straight into
// the matrix instructions' registers, and bound the time.  Internal; instantiated once per array type (ffn_few_*.hip).
//
// A work-group takes NR rows of the weights (NR of the gate's and the same NR of the up projection's) and all rows of
// x; its waves take blocks of k in turn, with the next block's loads in flight, and add their sums through LDS in a
// fixed order.  Weights and x may start on any element.
//
// A load takes 16 weight rows of 64 bytes, the 16 x 16 instruction's operand, or, for more work-groups and whole lines
// (NR = 8), 8 rows of 128: lane l has row l & 7 and 16-byte chunk (l >> 4) + 4 (l >> 3 & 1), eight rows twice, the second
// time at the other half of k; it is multiplied by x at either half, and of the two results the first gives rows 0 - 7
// and the second rows 8 - 15.  16-bit arrays run on the 16 x 16 x 32 instruction, 32-bit ones on the 32-bit 16 x 16 x 4:
// four of those take a lane's 16 bytes, element j of every lane as one k set.  One bf16 row reads 16384 x 4096 gated
// weights at 5.5 TB/s, 2048 x 8192 ones at 3.5.
#pragma once

#include "ffn_tile.h"

namespace ffn {
namespace dev {

template <typename T> struct Few {                       // 16 bytes of a row
    static constexpr int kPer = 16 / (int)sizeof(T), kChunk = 4 * kPer;   // values a lane, k of four lanes
    typedef T V __attribute__((ext_vector_type(kPer)));
};
__device__ __forceinline__ f32x4 few_mfma(Few<bf16>::V a, Few<bf16>::V b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 few_mfma(Few<fp16>::V a, Few<fp16>::V b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 few_mfma(Few<float>::V a, Few<float>::V b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
}

// MT: tiles of 16 rows of x.  EPI: kGate or kStore.
template <typename T, int MT, int NR, int EPI>
__global__ __launch_bounds__(512) void few_kernel(FewArgs p) {
#ifdef __HIP_DEVICE_COMPILE__
    typedef typename Few<T>::V V;
    constexpr int kPer = Few<T>::kPer, kChunk = Few<T>::kChunk, HB = NR == 8 ? 2 : 1, kStep = HB * kChunk;
    constexpr int kRows = 16 / HB, RT = NR / kRows, G = EPI == kGate ? 2 : 1, F = RT * G, U = F * MT * HB <= 2 ? 4 : F * MT * HB <= 8 ? 2 : 1;
    constexpr int kBlock = U * kStep;
    extern __shared__ f32x4 few_sums[];                  // [waves][tiles][64]
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    const int64_t n0 = (int64_t)blockIdx.x * NR;
    const int K = (int)p.K, q = (lane >> 4) * kPer, qw = q + (HB == 2 ? (lane >> 3 & 1) * kChunk : 0);

    const T *w[F], *x[MT];
#pragma unroll
    for (int f = 0; f < F; ++f) {
        int64_t n = n0 + (f % RT) * kRows + (lane & (kRows - 1));
        if (n >= p.N) n = p.N - 1;
        w[f] = (const T*)p.w + (n + (f / RT) * p.N) * p.ldw;
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        int64_t r = m * 16 + (lane & 15);
        if (r >= p.M) r = p.M - 1;
        x[m] = (const T*)p.x + r * p.ldx;
    }

    f32x4 acc[F][MT][HB] = {};
    V wf[2][U][F], xf[2][U][MT][HB];
    auto fetch = [&](int to, int k0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int f = 0; f < F; ++f) __builtin_memcpy(&wf[to][u][f], w[f] + k0 + u * kStep + qw, 16);
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int b = 0; b < HB; ++b) __builtin_memcpy(&xf[to][u][m][b], x[m] + k0 + u * kStep + q + b * kChunk, 16);
        }
        __builtin_amdgcn_sched_barrier(0);   // all of them issued before the other block is multiplied
    };
    auto multiply = [&](int of) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int f = 0; f < F; ++f)
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int b = 0; b < HB; ++b) acc[f][m][b] = few_mfma(wf[of][u][f], xf[of][u][m][b], acc[f][m][b]);
    };
    // this wave's whole blocks, two in registers: the loop has no branch between a load and its use, so that the
    // compiler waits for the older block alone
    const int whole = K / kBlock, stride = waves * kBlock;
    int left = whole > wave ? (whole - wave + waves - 1) / waves : 0, k = wave * kBlock;
    if (left > 0) {
        fetch(0, k);
        for (; left > 2; left -= 2) {
            fetch(1, k + stride);
            multiply(0);
            k += 2 * stride;
            fetch(0, k);
            multiply(1);
        }
        if (left == 2) {
            fetch(1, k + stride);
            multiply(0);
            multiply(1);
        } else {
            multiply(0);
        }
    }
    if (whole * kBlock < K && wave == whole % waves) {
        // the rest of k, a load at a time; values beyond it are zeros on both sides
        for (int at = whole * kBlock; at < K; at += kStep) {
            auto part = [&](const T* from, int q) {
                V v = {};
                if (at + q + kPer <= K) {
                    __builtin_memcpy(&v, from + at + q, 16);
                } else {
#pragma unroll
                    for (int j = 0; j < kPer; ++j)
                        if (at + q + j < K) v[j] = from[at + q + j];
                }
                return v;
            };
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int b = 0; b < HB; ++b) xf[0][0][m][b] = part(x[m], q + b * kChunk);
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const V v = part(w[f], qw);
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int b = 0; b < HB; ++b) acc[f][m][b] = few_mfma(v, xf[0][0][m][b], acc[f][m][b]);
            }
        }
    }

    // acc[f][m][b][e] is weight row .. + 4 (lane / 16) + e (HB = 2: of lanes 32 b .. 32 b + 31, 4 (lane / 16 & 1)), row of x
    // .. + lane % 16
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
        for (int m = 0; m < MT; ++m)
            {
            const f32x4 lo = acc[f][m][0], hi = acc[f][m][HB - 1];
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = lane < 32 ? lo[e] : hi[e];
            few_sums[(wave * F * MT + f * MT + m) * 64 + lane] = HB == 1 ? lo : v;
            }
    __syncthreads();
    constexpr int kLanes = 64 / HB;
    for (int i = threadIdx.x; i < RT * MT * kLanes; i += blockDim.x) {
        const int l = i % kLanes, tile = i / kLanes, rt = tile / MT, mt = tile % MT;
        const int64_t r = mt * 16 + (l & 15), n = n0 + rt * kRows + (l >> 4) * 4;
        if (r >= p.M || n >= p.N) continue;
        f32x4 v = {}, u = {};
        for (int s = 0; s < waves; ++s) {
            const f32x4* t = few_sums + (s * F * MT + tile) * 64 + l;
#pragma unroll
            for (int b = 0; b < HB; ++b) {
                v += t[32 * b];
                if constexpr (EPI == kGate) u += t[RT * MT * 64 + 32 * b];
            }
        }
        if constexpr (EPI == kGate) {
            f32x4 h;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float a, da;
                activate<T>(p.act, v[e], a, da);
                h[e] = a * u[e];
            }
            store4<T>((T*)p.c + r * p.ldc, n, p.N, p.ldc, h);
            if (p.saved) {
                store4<float>(p.saved + r * 2 * p.N, n, p.N, 0, v);
                store4<float>(p.saved + r * 2 * p.N + p.N, n, p.N, 0, u);
            }
        } else {
            store4<T>((T*)p.c + r * p.ldc, n, p.N, 0, v);
        }
    }
#endif
}

template <typename T, int MT, int EPI> int run_few(const FewArgs& p, int nr, int waves, hipStream_t s) {
    const dim3 grid((unsigned)((p.N + nr - 1) / nr));
    const int tiles = (nr > 16 ? 2 : 1) * (EPI == kGate ? 2 : 1) * MT;
    const int lds = waves * tiles * 1024;
    if (lds > 64 * 1024) return (int)hipErrorInvalidValue;
    // (those that few_product() asks for)
    constexpr bool k16 = MT > 1 || sizeof(T) == 4, k32 = MT > 1 && EPI == kGate;
    if (nr == 8) {
        few_kernel<T, MT, 8, EPI><<<grid, waves * 64, lds, s>>>(p);
        return (int)hipGetLastError();
    }
    if constexpr (k16) {
        if (nr == 16) {
            few_kernel<T, MT, 16, EPI><<<grid, waves * 64, lds, s>>>(p);
            return (int)hipGetLastError();
        }
    }
    if constexpr (k32) {
        if (nr == 32) {
            few_kernel<T, MT, 32, EPI><<<grid, waves * 64, lds, s>>>(p);
            return (int)hipGetLastError();
        }
    }
    return (int)hipErrorInvalidValue;
}

template <typename T> int few(const FewArgs& p, int32_t epilogue, int nr, int waves, hipStream_t s) {
    const int mt = p.M <= 16 ? 1 : p.M <= 32 ? 2 : 4;
    if (epilogue == kGate)
        return mt == 1 ? run_few<T, 1, kGate>(p, nr, waves, s) : mt == 2 ? run_few<T, 2, kGate>(p, nr, waves, s) : run_few<T, 4, kGate>(p, nr, waves, s);
    return mt == 1 ? run_few<T, 1, kStore>(p, nr, waves, s) : mt == 2 ? run_few<T, 2, kStore>(p, nr, waves, s) : run_few<T, 4, kStore>(p, nr, waves, s);
}

}  // namespace dev
}  // namespace ffn
