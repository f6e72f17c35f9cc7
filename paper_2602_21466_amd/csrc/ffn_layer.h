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

// r from the sum of the centred values' squares.  NaN stays NaN (fmaxf would drop it), and a variance past the range of 32 bits
// infinite, r = 0, also where d^2 passes it.
__device__ __forceinline__ float layer_r(float s2, float d, float D, float eps) {
    const float v = s2 / D - fminf(d * d, 3.4028235e38f);
    return 1.0f / sqrtf((v < 0.0f ? 0.0f : v) + eps);
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
        const float r = layer_r(group_sum(s2, s), d, (float)D, p.eps);
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

// A worker of TPR threads holds a row in registers, eight adjacent columns a thread and turn (as the norms of ffn_norm.h),
// with the next row's loads in flight: x is read and u written once.  Bound by memory (16384 x 4096 in bf16: 50 us, 5.4
// TB/s; with the backward pass 146, 214 by kernels that read rows again), with few rows by their latency (4001 x 1089 in fp16:
// 9.2 us).
template <typename T, int TPR, int I, bool TAIL>
__global__ __launch_bounds__(group_of(TPR), forward_waves(sizeof(T), TPR, I, false)) void layer_forward_rows(LayerArgs p) {
    __shared__ float s[4 * (TPR > 64 ? TPR / 64 : 1)];
    constexpr int kWorkers = group_of(TPR) / TPR;
    typedef Eight<T> V;
    const int D = (int)p.width, t = threadIdx.x % TPR;
    const int64_t step = (int64_t)gridDim.x * kWorkers;
    const int sub = kWorkers == 1 ? 0 : TPR < 64 ? threadIdx.x / TPR : __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    int64_t row = (int64_t)blockIdx.x * kWorkers + sub;
    if (row >= p.N) return;
    V w[I], b[I], xr[I];
    Place at8[I];
#pragma unroll
    for (int i = 0; i < I; ++i) at8[i] = place8<TAIL>((t + i * TPR) * 8, D);
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int i = 0; i < I; ++i) xr[i] = row8<T>((const T*)p.x + r * p.ldx, at8[i]);
    };
    auto factors = [&](int i) {
        w[i] = ones8<T>(p.w, at8[i]);
        b[i] = p.b ? row8<T>((const T*)p.b, at8[i]) : V{};
    };
    constexpr bool kLean = TPR == 1024;   // (128 registers a thread: neither the next row nor the factors are held)
    if constexpr (!kLean) {
        fetch(row);
#pragma unroll
        for (int i = 0; i < I; ++i) factors(i);
    }
    for (; row < p.N; row += step) {
#pragma unroll
        for (int i = 0; i < I; ++i) {   // neither lanes' addresses nor converted factors are held over the rows
            if constexpr (!kLean) {
                asm volatile("" : "+v"(at8[i].c));
                keep(w[i]);
                keep(b[i]);
            }
        }
        if constexpr (kLean) fetch(row);
        float v[I][8], one[1] = {0.0f}, two[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < I; ++i) {
            if constexpr (TAIL) keep(xr[i]);   // here before another thread may write u over it
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[i][j] = at(xr[i], j);
                one[0] += (TAIL ? j >= at8[i].skip : at8[i].skip == 0) ? v[i][j] : 0.0f;
            }
        }
        if (!kLean && row + step < p.N) fetch(row + step);
        worker_sum<TPR, 1>(one, s, 0);
        const float m = one[0] / (float)D;
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[i][j] -= m;
                const float c = (TAIL ? j >= at8[i].skip : at8[i].skip == 0) ? v[i][j] : 0.0f;
                two[0] += c;
                two[1] += c * c;
            }
        worker_sum<TPR, 2>(two, s, 1);
        const float d = two[0] / (float)D, r = layer_r(two[1], d, (float)D, p.eps);
        if (p.stats && t == 0) {
            p.stats[row] = m + d;
            p.stats[p.N + row] = r;
        }
#pragma unroll
        for (int i = 0; i < I; ++i) {
            float o[8];
            if constexpr (kLean) factors(i);
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = (v[i][j] - d) * r * at(w[i], j) + at(b[i], j);
            if (at8[i].skip < 8) put8<T>((T*)p.u + row * p.ldu, at8[i], o);
        }
    }
}

// Waves a SIMD that the backward rows' registers are bounded for: two column sums a value live through the rows.  Two turns of
// 32-bit values take 173 registers, which is two waves (in fp32 16384 x 2500: 97 us; by three, with registers in scratch memory, 161,
// and with w loaded twice a row instead 117; 8192 x 4096: 81, 103 and 90).
constexpr int layer_backward_waves(int bytes, int tpr, int turns) { return turns == 1 || tpr == 1024 || bytes == 2 ? 4 : 2; }

// One pass over the rows: gx, and each work-group's column sums, which stay in registers.  (16384 x 4096 in bf16: 88 us, 4.9
// TB/s, and 7.5 for the joining of 1024 sets; 4001 x 1089 in fp16: 14.2 and 6.2.)
template <typename T, int TPR, int I, bool TAIL>
__global__ __launch_bounds__(group_of(TPR), layer_backward_waves(sizeof(T), TPR, I)) void layer_backward_rows(LayerArgs p, int64_t workers) {
    constexpr int kGroup = group_of(TPR), kWorkers = kGroup / TPR;
    __shared__ float s[2 * 3 * (TPR > 64 ? TPR / 64 : 1)];
    __shared__ float cols[kWorkers > 1 ? kWorkers * TPR * I * 8 : 1];
    typedef Eight<T> V;
    const int D = (int)p.width, t = threadIdx.x % TPR;
    const int sub = kWorkers == 1 ? 0 : TPR < 64 ? threadIdx.x / TPR : __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    const int64_t worker = (int64_t)blockIdx.x * kWorkers + sub;
    int64_t row = worker < workers ? worker : p.N;
    float sw[I][8] = {}, sb[I][8] = {}, mr = 0.0f, rr = 0.0f;
    V xr[I], gr[I], w[I];
    Place at8[I];
#pragma unroll
    for (int i = 0; i < I; ++i) at8[i] = place8<TAIL>((t + i * TPR) * 8, D);
    auto fetch = [&](int64_t r) {
        mr = p.stats[r];
        rr = p.stats[p.N + r];
#pragma unroll
        for (int i = 0; i < I; ++i) {
            xr[i] = row8<T>((const T*)p.x + r * p.ldx, at8[i]);
            gr[i] = row8<T>((const T*)p.gu + r * p.ldg, at8[i]);
        }
    };
    // (kAgain: nor is w held from the sums to gx, as 128 registers do not hold it beside 32-bit values; 4096 x 16384 in fp32: 175
    // us, 210 with registers in scratch memory)
    constexpr bool kLean = TPR == 1024, kAgain = kLean && sizeof(T) == 4;
    if constexpr (!kLean) {
        if (row < p.N) fetch(row);
#pragma unroll
        for (int i = 0; i < I; ++i) w[i] = ones8<T>(p.w, at8[i]);
    }
    for (int turn = 0; row < p.N; turn ^= 1) {
#pragma unroll
        for (int i = 0; i < I; ++i) asm volatile("" : "+v"(at8[i].c), "+v"(at8[i].skip));
        if constexpr (kLean) fetch(row);
        const float m = mr, r = rr;
        V x[I], g[I];
        float sum[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < I; ++i) {
            if constexpr (kLean) w[i] = ones8<T>(p.w, at8[i]);
            x[i] = xr[i];
            g[i] = gr[i];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool own = TAIL ? j >= at8[i].skip : at8[i].skip == 0;
                const float a = own ? at(g[i], j) * at(w[i], j) : 0.0f, c = own ? at(x[i], j) - m : 0.0f;
                sum[0] += a;
                sum[1] += c;
                sum[2] += a * c;
            }
            keep(x[i]);   // the next half starts from the loaded values
            keep(g[i]);
            if constexpr (!kAgain) keep(w[i]);
        }
        const int64_t at_row = row;
        row += workers;
        if (!kLean && row < p.N) fetch(row);
        worker_sum<TPR, 3>(sum, s, turn);
        const float ma = sum[0] / (float)D, d = sum[1] / (float)D, man = r * (sum[2] / (float)D - d * ma);
#pragma unroll
        for (int i = 0; i < I; ++i) {
            if (at8[i].skip == 8) continue;
            if constexpr (kAgain) {
                asm volatile("" : "+v"(at8[i].c));
                w[i] = ones8<T>(p.w, at8[i]);
            }
            float gx[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float gu = at(g[i], j), n = (at(x[i], j) - m - d) * r;
                sw[i][j] += gu * n;
                sb[i][j] += gu;
                gx[j] = r * (gu * at(w[i], j) - ma - n * man);
            }
            if (p.gx) put8<T>((T*)p.gx + at_row * D, at8[i], gx);
        }
    }

    // column sums of the work-group
    float* out = p.partial + (int64_t)blockIdx.x * 2 * D;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if constexpr (kWorkers > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (at8[i].skip < 8) cols[sub * (TPR * I * 8) + at8[i].c + j] = k ? sb[i][j] : sw[i][j];
            __syncthreads();
            for (int c = threadIdx.x; c < D; c += kGroup) {
                float v = 0.0f;
#pragma unroll
                for (int q = 0; q < kWorkers; ++q) v += cols[q * (TPR * I * 8) + c];
                out[(int64_t)k * D + c] = v;
            }
        } else {
#pragma unroll
            for (int i = 0; i < I; ++i) {
                if (at8[i].skip == 8) continue;
#pragma unroll
                for (int j = 0; j < 8; ++j) out[(int64_t)k * D + at8[i].c + j] = k ? sb[i][j] : sw[i][j];
            }
        }
    }
}

// Workers of the backward pass: as many as the compute units hold at once, with two or four rows each where there are many
// (the joining kernel reads a set of sums for each work-group).
inline int64_t layer_workers(const Shape& sh, int64_t N, int64_t width, int bytes) {
    const int64_t least = N >= 4096 ? 4 : N >= 256 ? 2 : 1, some = (N + least - 1) / least;
    int64_t most = 1024 / column_blocks(width);
    if (sh.tpr) most = 256 * (256 * layer_backward_waves(bytes, sh.tpr, sh.turns) / group_of(sh.tpr)) * (group_of(sh.tpr) / sh.tpr);
    if (most < 1) most = 1;
    return some < most ? some : most;
}
inline int64_t layer_groups(const Shape& sh, int64_t workers) {
    const int64_t per = sh.tpr ? group_of(sh.tpr) / sh.tpr : 1;
    return (workers + per - 1) / per;
}

template <typename T> int layer_forward(const LayerArgs& a, hipStream_t s) {
    const Shape sh = shape_of(a.width, kForward, (int)sizeof(T));
    if (sh.tpr == 0) {
        layer_forward_kernel<T><<<dim3(row_groups(a.N)), kThreads, 0, s>>>(a);
        return (int)hipGetLastError();
    }
    const bool tail = a.width % 8 != 0;
    const int64_t per = group_of(sh.tpr) / sh.tpr, all = (a.N + per - 1) / per;
    const int64_t most = 256 * (256 * forward_waves(sizeof(T), sh.tpr, sh.turns, false) / group_of(sh.tpr));
    const dim3 grid((unsigned)(all < most ? all : most));
#define FFN_RUN(TPR, I)                                                                  \
    if (tail) layer_forward_rows<T, TPR, I, true><<<grid, group_of(TPR), 0, s>>>(a);     \
    else layer_forward_rows<T, TPR, I, false><<<grid, group_of(TPR), 0, s>>>(a)
    FFN_SHAPES(FFN_RUN)
#undef FFN_RUN
    return (int)hipGetLastError();
}

template <typename T> int layer_backward(const LayerArgs& a, hipStream_t s) {
    const Shape sh = shape_of(a.width, kBackward, (int)sizeof(T));
    const int64_t workers = layer_workers(sh, a.N, a.width, (int)sizeof(T)), groups = layer_groups(sh, workers);
    if (groups > 0 && sh.tpr == 0) {
        layer_means_kernel<T><<<dim3(row_groups(a.N)), kThreads, 0, s>>>(a, groups);
        layer_columns_kernel<T><<<dim3((unsigned)groups, (unsigned)column_blocks(a.width)), kThreads, 0, s>>>(a, groups);
    } else if (groups > 0) {
        const bool tail = a.width % 8 != 0;
        const dim3 grid((unsigned)groups);
#define FFN_RUN(TPR, I)                                                                           \
    if (tail) layer_backward_rows<T, TPR, I, true><<<grid, group_of(TPR), 0, s>>>(a, workers);    \
    else layer_backward_rows<T, TPR, I, false><<<grid, group_of(TPR), 0, s>>>(a, workers)
        FFN_SHAPES(FFN_RUN)
#undef FFN_RUN
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

inline int64_t layer_floats(int64_t width, int64_t N, int bytes) {
    const Shape sh = shape_of(width, kBackward, bytes);
    return layer_groups(sh, layer_workers(sh, N, width, bytes)) * 2 * width + (sh.tpr ? 0 : 3 * N);
}

}  // namespace
}  // namespace ffn
