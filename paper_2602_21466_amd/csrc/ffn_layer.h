// Kernels of the layer norm.  Internal; instantiated once per array type (ffn_layer_*.hip).
//
// The mean m is a 32-bit sum and rounded, by up to 2^-24 |m|, which is not small beside the values' spread where they lie
// far from zero.  So the centred values c = x - m are summed again, with their squares: d = mean(c) is what m lacks, and
// n = (c - d) r with r = 1 / sqrt(mean(c^2) - d^2 + eps).  The backward pass, given m and r, takes d from the same pass as
// its own sums: mean(a) and mean(a n) = r (mean(a c) - d mean(a)).
#pragma once

#include "experts_internal.h"
#include "ffn_norm.h"

namespace ffn {
namespace {

using namespace dev;

template <typename T> __device__ __forceinline__ void offsets8(const void* p, int64_t c, int64_t D, float (&f)[8]) {
    if (p) {
        factors8<T>(p, c, D, f);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = 0.0f;
    }
}

// One row a work-group, eight columns a thread and turn, any width: a row is read three times, from the caches while it
// fits them.
template <typename T>
__global__ __launch_bounds__(kThreads) void layer_forward_kernel(LayerArgs p) {
    __shared__ float s[kThreads / 64];
    const int64_t D = p.width;
    for (int64_t row = blockIdx.x; row < p.N; row += gridDim.x) {
        const T* x = (const T*)p.x + row * p.ldx;
        float sum = 0.0f;
        for (int64_t c = threadIdx.x * 8; c < D; c += kThreads * 8) {
            float v[8];
            factors8<T>(x, c, D, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += v[j];   // (zeros beyond the row)
        }
        const float m = group_sum(sum, s) / (float)D;
        float s1 = 0.0f, s2 = 0.0f;
        for (int64_t c = threadIdx.x * 8; c < D; c += kThreads * 8) {
            float v[8];
            factors8<T>(x, c, D, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = c + j < D ? v[j] - m : 0.0f;
                s1 += v[j];
                s2 += v[j] * v[j];
            }
        }
        const float d = group_sum(s1, s) / (float)D;
        const float r = 1.0f / sqrtf(fmaxf(group_sum(s2, s) / (float)D - d * d, 0.0f) + p.eps);
        if (p.stats && threadIdx.x == 0) {
            p.stats[row] = m + d;
            p.stats[p.N + row] = r;
        }
        for (int64_t c = threadIdx.x * 8; c < D; c += kThreads * 8) {
            float v[8], w[8], b[8];
            factors8<T>(x, c, D, v);
            factors8<T>(p.w, c, D, w);
            offsets8<T>(p.b, c, D, b);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = (v[j] - m - d) * r * w[j] + b[j];
            store8((T*)p.u + row * p.ldu, c, D, v);
        }
    }
}

// Rows too wide or too narrow for registers, backward: d, mean(a) and mean(a n) of each row first, behind the column sums.
template <typename T>
__global__ __launch_bounds__(kThreads) void layer_means_kernel(LayerArgs p, int64_t workers) {
    __shared__ float s[kThreads / 64];
    const int64_t D = p.width;
    float* means = p.partial + workers * 2 * D;
    for (int64_t row = blockIdx.x; row < p.N; row += gridDim.x) {
        const T *x = (const T*)p.x + row * p.ldx, *gu = (const T*)p.gu + row * p.ldg;
        const float m = p.stats[row], r = p.stats[p.N + row];
        float sa = 0.0f, sc = 0.0f, sac = 0.0f;
        for (int64_t c = threadIdx.x * 8; c < D; c += kThreads * 8) {
            float v[8], g[8], w[8];
            factors8<T>(x, c, D, v);
            factors8<T>(gu, c, D, g);
            factors8<T>(p.w, c, D, w);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + j < D) {
                    const float a = g[j] * w[j], e = v[j] - m;
                    sa += a;
                    sc += e;
                    sac += a * e;
                }
        }
        const float ma = group_sum(sa, s) / (float)D, d = group_sum(sc, s) / (float)D, mac = group_sum(sac, s) / (float)D;
        if (threadIdx.x == 0) {
            means[row] = d;
            means[p.N + row] = ma;
            means[2 * p.N + row] = r * (mac - d * ma);
        }
    }
}

// A thread eight columns of one worker's rows (the rows k, k + workers, ..): gx and the column sums.
template <typename T>
__global__ __launch_bounds__(kThreads) void layer_columns_kernel(LayerArgs p, int64_t workers) {
    const int64_t D = p.width, c = ((int64_t)blockIdx.y * kThreads + threadIdx.x) * 8, worker = blockIdx.x;
    if (c >= D) return;
    const float* means = p.partial + workers * 2 * D;
    float w[8], sw[8] = {}, sb[8] = {};
    factors8<T>(p.w, c, D, w);
    for (int64_t row = worker; row < p.N; row += workers) {
        const float m = p.stats[row], r = p.stats[p.N + row], d = means[row], ma = means[p.N + row], man = means[2 * p.N + row];
        float v[8], g[8];
        factors8<T>((const T*)p.x + row * p.ldx, c, D, v);
        factors8<T>((const T*)p.gu + row * p.ldg, c, D, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float n = (v[j] - m - d) * r;
            sw[j] += g[j] * n;
            sb[j] += g[j];
            v[j] = r * (g[j] * w[j] - ma - n * man);
        }
        if (p.gx) store8((T*)p.gx + row * D, c, D, v);
    }
    float* out = p.partial + worker * 2 * D + c;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (c + j < D) {
            out[j] = sw[j];
            out[D + j] = sb[j];
        }
}

inline int64_t layer_workers(int64_t width, int64_t N) {
    const int64_t most = 1024 / column_blocks(width), least = N >= 256 ? N / 2 : N;
    return N == 0 ? 0 : most < 1 ? 1 : most < least ? most : least;
}

template <typename T> int layer_forward(const LayerArgs& a, hipStream_t s) {
    layer_forward_kernel<T><<<dim3(row_groups(a.N)), kThreads, 0, s>>>(a);
    return (int)hipGetLastError();
}

template <typename T> int layer_backward(const LayerArgs& a, hipStream_t s) {
    const int64_t groups = layer_workers(a.width, a.N);
    if (groups > 0) {
        layer_means_kernel<T><<<dim3(row_groups(a.N)), kThreads, 0, s>>>(a, groups);
        layer_columns_kernel<T><<<dim3((unsigned)groups, (unsigned)column_blocks(a.width)), kThreads, 0, s>>>(a, groups);
    }
    if (a.gw || a.gb) {
        // the work-groups' sums added by the norms' joining kernel
        NormArgs n = {};
        n.width = a.width;
        n.gw = a.gw;
        n.gwn = a.gb;
        n.partial = a.partial;
        const Join jn = {2, 5, 0};
        norm_join_kernel<T><<<dim3((unsigned)(2 * ((a.width + 31) / 32))), 1024, 0, s>>>(n, Rows{1, groups}, groups, jn);
    }
    return (int)hipGetLastError();
}

inline int64_t layer_floats(int64_t width, int64_t N, int bytes) { (void)bytes; return layer_workers(width, N) * 2 * width + 3 * N; }

}  // namespace
}  // namespace ffn
