// Gradients of the feed-forward block for few rows of 32-bit arrays: C = A W with W stored [K, N], which is read once
// and bounds the time (14320 x 3464, 5 rows: 40 us, 5.0 TB/s).
//
// A work-group takes 64 columns and a part of k; its waves take 16 k in turn.  A load is four rows of 256 bytes: lane l
// has row 4 (l / 16) + t of the 16 and columns 4 (l % 16) .. + 3, and x's values of the same k, so that element j of all
// lanes is an operand of the 16 x 16 x 4 instruction for columns 4 i + j.  Waves are added through LDS and work-groups
// by the joining kernel, both in a fixed order.
#include "ffn_tile.h"

namespace ffn {
namespace {

using namespace dev;

template <int MT>
__global__ __launch_bounds__(512) void few_grad_kernel(FewGradArgs p) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int U = MT <= 2 ? 2 : 1;
    extern __shared__ f32x4 sums[];   // [waves][4][MT][64]
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    const int N = (int)p.N, K = (int)p.K, n0 = (int)blockIdx.x * 64, q = lane >> 4, i = lane & 15;
    // columns that would pass the last one are the last four once more (N >= 4): the same sums, stored twice
    const int nc = n0 + 4 * i + 4 <= N ? n0 + 4 * i : N - 4;
    const float* w = (const float*)p.w + nc;
    int64_t xr[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        int64_t r = m * 16 + i;
        if (r >= p.M) r = p.M - 1;
        xr[m] = r * p.ldx;
    }
    f32x4 acc[4][MT] = {}, wf[2][U][4], xf[2][U][MT];
    auto load_x = [&](int m, int k) {
        f32x4 v = {};
        __builtin_memcpy(&v, (const float*)p.x + xr[m] + k, sizeof(v));
        return v;
    };
    auto fetch = [&](int to, int k0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = k0 + u * 16 + q * 4;
#pragma unroll
            for (int t = 0; t < 4; ++t) __builtin_memcpy(&wf[to][u][t], w + (int64_t)(k + t) * p.ldw, 16);
#pragma unroll
            for (int m = 0; m < MT; ++m) xf[to][u][m] = load_x(m, k);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto multiply = [&](int of) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int m = 0; m < MT; ++m)
                        acc[j][m] = __builtin_amdgcn_mfma_f32_16x16x4f32(wf[of][u][t][j], xf[of][u][m][t], acc[j][m], 0, 0, 0);
    };
    // this wave's whole blocks of 16 U k, two in registers
    constexpr int kBlock = 16 * U;
    const int slices = waves * p.splits, slice = (int)blockIdx.y * waves + wave, whole = K / kBlock, stride = slices * kBlock;
    int left = whole > slice ? (whole - slice + slices - 1) / slices : 0, k = slice * kBlock;
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
    if (whole * kBlock < K && slice == whole % slices) {
        // the rest of k, four a lane group and turn; values beyond it are zeros on both sides
        for (int k0 = whole * kBlock; k0 < K; k0 += 16) {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int kt = k0 + q * 4 + t;
                f32x4 wv = {};
                if (kt < K) __builtin_memcpy(&wv, w + (int64_t)kt * p.ldw, 16);
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    float xv = 0.0f;
                    if (kt < K) xv = ((const float*)p.x)[xr[m] + kt];
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[j][m] = __builtin_amdgcn_mfma_f32_16x16x4f32(wv[j], xv, acc[j][m], 0, 0, 0);
                }
            }
        }
    }
    // acc[j][m][e] of lane l: columns 4 (4 (l / 16) + e) + j, row of x l % 16
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int m = 0; m < MT; ++m) sums[((wave * 4 + j) * MT + m) * 64 + lane] = acc[j][m];
    __syncthreads();
    for (int s = threadIdx.x; s < MT * 64; s += blockDim.x) {
        const int l = s & 63, m = s >> 6, r = m * 16 + (l & 15);
        if (r >= p.M) continue;
        f32x4 v[4] = {};
        for (int u = 0; u < waves; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] += sums[((u * 4 + j) * MT + m) * 64 + l];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int c = n0 + 4 * (4 * (l >> 4) + e), at = c + 4 <= N ? c : N - 4;
            const f32x4 o = {v[0][e], v[1][e], v[2][e], v[3][e]};
            __builtin_memcpy(p.c + ((int64_t)blockIdx.y * p.M + r) * p.ldc + at, &o, sizeof(o));
        }
    }
#endif
}

int run(const FewGradArgs& p, hipStream_t s) {
    const dim3 grid((unsigned)((p.N + 63) / 64), (unsigned)p.splits);
    const int mt = p.M <= 16 ? 1 : p.M <= 32 ? 2 : 4, lds = p.waves * 4 * mt * 1024;
    if (lds > 64 * 1024 || p.N < 4 || p.M > 64) return (int)hipErrorInvalidValue;
    if (mt == 1) few_grad_kernel<1><<<grid, p.waves * 64, lds, s>>>(p);
    else if (mt == 2) few_grad_kernel<2><<<grid, p.waves * 64, lds, s>>>(p);
    else few_grad_kernel<4><<<grid, p.waves * 64, lds, s>>>(p);
    return (int)hipGetLastError();
}

}  // namespace

int launch_few_grad(const FewGradArgs& p, void* stream) {
    return run(p, (hipStream_t)stream);
}

}  // namespace ffn
