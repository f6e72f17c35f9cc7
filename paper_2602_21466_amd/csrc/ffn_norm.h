// Kernels of the norms before and after a block with its gate and residual scale, and of dropout.  Internal;
// instantiated once per array type (ffn_norm_*.hip).
#pragma once

#include "ffn_device.h"

namespace ffn {
namespace {

using namespace dev;

constexpr int kThreads = 256;

template <typename T> __device__ __forceinline__ float load(const void* p, int64_t i, float missing) {
    return p ? to_f32(((const T*)p)[i]) : missing;
}

// Dropout factor of (row, column).
__device__ __forceinline__ float factor(const DropArgs& d, int64_t row, int64_t c) {
    if (d.threshold == 0) return 1.0f;
    const Words q = philox((uint32_t)(c >> 3), (uint32_t)row, d.offset, d.seed);
    return kept(q, (int)(c & 7), d.threshold) ? d.scale : 0.0f;
}

// One row a work-group: y = x + scale * gate * drop(N(h; w)) where h is given, then u = N(y; wn).
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_forward_kernel(NormArgs p) {
    __shared__ float s[kThreads / 64];
    const int64_t D = p.width;
    for (int64_t row = blockIdx.x; row < p.N; row += gridDim.x) {
    const T* x = (const T*)p.x + row * p.ldx;
    const T* h = p.h ? (const T*)p.h + row * D : nullptr;
    float rh = 0.0f;
    if (h) {
        float sum = 0.0f;
        for (int64_t c = threadIdx.x; c < D; c += kThreads) sum += to_f32(h[c]) * to_f32(h[c]);
        rh = 1.0f / sqrtf(group_sum(sum, s) / (float)D + p.eps);
        if (p.rstd_h && threadIdx.x == 0) p.rstd_h[row] = rh;
    }
    const int64_t gate = row / p.rows_per_gate * D;
    auto joined = [&](int64_t c) {
        float v = to_f32(x[c]);
        if (h) {
            const float f = factor(p.drop, row, c);
            const float n = to_f32(h[c]) * rh * load<T>(p.w, c, 1.0f);
            const float b = f == 0.0f ? 0.0f : n * f;
            v += load<T>(p.scale, c, 1.0f) * load<T>(p.gate, gate + c, 1.0f) * b;
        }
        return v;
    };
    if (p.u) {
        float sum = 0.0f;
        for (int64_t c = threadIdx.x; c < D; c += kThreads) { const float v = joined(c); sum += v * v; }
        const float ry = 1.0f / sqrtf(group_sum(sum, s) / (float)D + p.eps);
        if (p.rstd_y && threadIdx.x == 0) p.rstd_y[row] = ry;
        for (int64_t c = threadIdx.x; c < D; c += kThreads) {
            const float v = joined(c);
            if (p.y) ((T*)p.y)[row * D + c] = (T)v;
            ((T*)p.u)[row * p.ldu + c] = (T)(v * ry * load<T>(p.wn, c, 1.0f));
        }
    } else {
        for (int64_t c = threadIdx.x; c < D; c += kThreads) ((T*)p.y)[row * D + c] = (T)joined(c);
    }
    }
}

// ---------------------------------------------------------------- rows held in registers
//
// A worker of TPR threads takes a row, eight adjacent values (one block of the generator) a thread and turn, I turns:
// every array is read and written once, and the row's sums stay in registers.  Workers of 64 threads or fewer reduce by
// shuffles alone; a wider worker is a work-group and passes its waves' sums through LDS.

template <typename T> struct Raw { typedef T V __attribute__((ext_vector_type(8))); };

// Values c .. c + 7 of a row of D (zeros beyond it).  Rows may start on any element.
template <typename T> __device__ __forceinline__ typename Raw<T>::V load8(const T* row, int64_t c, int64_t D) {
    typename Raw<T>::V v;
    if (c + 8 <= D) {
        __builtin_memcpy(&v, row + c, sizeof(v));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < D ? row[c + j] : (T)0.0f;
    }
    return v;
}
template <typename T> __device__ __forceinline__ void store8(T* row, int64_t c, int64_t D, const float (&f)[8]) {
    if (c + 8 <= D) {
        typename Raw<T>::V v;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (T)f[j];
        __builtin_memcpy(row + c, &v, sizeof(v));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j < D) row[c + j] = (T)f[j];
    }
}
// A row of factors; ones where there is none.
template <typename T> __device__ __forceinline__ void factors8(const void* p, int64_t c, int64_t D, float (&f)[8]) {
    if (p) {
        const typename Raw<T>::V v = load8((const T*)p, c, D);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = to_f32(v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = 1.0f;
    }
}
__device__ __forceinline__ void drop8(const DropArgs& d, int64_t row, int64_t c, float (&f)[8]) {
    if (d.threshold == 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = 1.0f;
        return;
    }
    const Words q = philox((uint32_t)(c >> 3), (uint32_t)row, d.offset, d.seed);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = kept(q, j, d.threshold) ? d.scale : 0.0f;
}

// Sums of K values over a worker, returned to all its threads.  `s` is LDS for two calls in turn (`turn` alternates):
// one barrier a call keeps both the values and the next but one call's writes in order.
template <int TPR, int K> __device__ __forceinline__ void worker_sum(float (&v)[K], float* s, int turn) {
#pragma unroll
    for (int o = (TPR < 64 ? TPR : 64) / 2; o; o >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += __shfl_xor(v[k], o, 64);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        float* t = s + turn * W * K;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) t[(threadIdx.x >> 6) * K + k] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float a = t[k];
#pragma unroll
            for (int w = 1; w < W; ++w) a += t[w * K + k];
            v[k] = a;
        }
    }
}

// Values c .. c + 7 of a row of D >= 8 (zeros beyond it).  TAIL: D is no multiple of 8; the last thread reads the
// row's last eight values and moves them down, so that no lane reads beside the row and no load is by single values.
template <typename T, bool TAIL> __device__ __forceinline__ typename Raw<T>::V row8(const T* row, int c, int D) {
    typename Raw<T>::V v = {};
    if (c < D) {
        const int at = TAIL && c > D - 8 ? D - 8 : c;
        __builtin_memcpy(&v, row + at, sizeof(v));
        if constexpr (TAIL) {
            const int by = c - at;
            if (by) {
                constexpr int W = sizeof(v) / 4;
                typedef uint32_t U __attribute__((ext_vector_type(W)));
                U u = __builtin_bit_cast(U, v);
#pragma unroll
                for (int b = 4; b; b >>= 1) {
                    const bool move = by & b;
                    const int words = b * (int)sizeof(T) / 4;
#pragma unroll
                    for (int k = 0; k < W; ++k) {
                        const uint32_t next = words ? (k + words < W ? u[k + words < W ? k + words : 0] : 0u)
                                                    : (u[k] >> 16 | (k + 1 < W ? u[k + 1 < W ? k + 1 : 0] << 16 : 0u));
                        u[k] = move ? next : u[k];
                    }
                }
                v = __builtin_bit_cast(typename Raw<T>::V, u);
            }
        }
    }
    return v;
}
template <typename T, bool TAIL> __device__ __forceinline__ void put8(T* row, int c, int D, const float (&f)[8]) {
    if (!TAIL || c + 8 <= D) {
        typename Raw<T>::V v;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (T)f[j];
        __builtin_memcpy(row + c, &v, sizeof(v));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j < D) row[c + j] = (T)f[j];
    }
}
// A row of factors, ones where there is none.
template <typename T, bool TAIL> __device__ __forceinline__ typename Raw<T>::V ones8(const void* p, int c, int D) {
    if (p) return row8<T, TAIL>((const T*)p, c, D);
    typename Raw<T>::V v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (T)1.0f;
    return v;
}

constexpr int group_of(int tpr) { return tpr > 64 ? tpr : 256; }

// BLOCK: y = x + scale gate drop(N(h; w)) first.  A worker walks its rows with the next one's loads in flight, the
// factors shared by all rows in registers; workers of 1024 threads have 128 registers each and do neither.
template <typename T, int TPR, int I, bool TAIL, bool BLOCK>
__global__ __launch_bounds__(group_of(TPR)) void norm_forward_rows(NormArgs p) {
    __shared__ float s[2 * (TPR > 64 ? TPR / 64 : 1)];
    constexpr int kWorkers = group_of(TPR) / TPR, B = BLOCK ? I : 1;
    typedef typename Raw<T>::V V;
    const int D = (int)p.width, t = threadIdx.x % TPR;
    const int64_t step = (int64_t)gridDim.x * kWorkers;
    int64_t row = (int64_t)blockIdx.x * kWorkers + threadIdx.x / TPR;
    if (row >= p.N) return;
    V wn[I], w[B], sc[B], xr[I], hr[B], gr[B];
    auto fetch = [&](int64_t r) {
        const T* gate = BLOCK && p.gate ? (const T*)p.gate + (int64_t)((uint32_t)r / (uint32_t)p.rows_per_gate) * D : nullptr;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int c = (t + i * TPR) * 8;
            xr[i] = row8<T, TAIL>((const T*)p.x + r * p.ldx, c, D);
            if constexpr (BLOCK) {
                hr[i] = row8<T, TAIL>((const T*)p.h + r * D, c, D);
                gr[i] = ones8<T, TAIL>(gate, c, D);
            }
        }
    };
    constexpr bool kLean = TPR == 1024;
    auto factors = [&](int i) {
        const int c = (t + i * TPR) * 8;
        wn[i] = ones8<T, TAIL>(p.wn, c, D);
        if constexpr (BLOCK) {
            w[i] = ones8<T, TAIL>(p.w, c, D);
            sc[i] = ones8<T, TAIL>(p.scale, c, D);
        }
    };
    if constexpr (!kLean) {
        fetch(row);
#pragma unroll
        for (int i = 0; i < I; ++i) factors(i);
    }
    for (int turn = 0; row < p.N; row += step) {
        if constexpr (kLean) fetch(row);
        float v[I][8];
        V h[B], g[B];
#pragma unroll
        for (int i = 0; i < I; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = to_f32(xr[i][j]);
            if constexpr (BLOCK) {
                h[i] = hr[i];
                g[i] = gr[i];
            }
        }
        if (!kLean && row + step < p.N) fetch(row + step);
        if constexpr (BLOCK) {
            float sum[1] = {0.0f};
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[0] += to_f32(h[i][j]) * to_f32(h[i][j]);
            worker_sum<TPR, 1>(sum, s, turn);
            turn ^= 1;
            const float rh = 1.0f / sqrtf(sum[0] / (float)D + p.eps);
            if (p.rstd_h && t == 0) p.rstd_h[row] = rh;
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const int c = (t + i * TPR) * 8;
                float f[8];
                drop8(p.drop, row, c, f);
                if constexpr (kLean) factors(i);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float n = to_f32(h[i][j]) * rh * to_f32(w[i][j]);
                    v[i][j] += to_f32(sc[i][j]) * to_f32(g[i][j]) * (f[j] == 0.0f ? 0.0f : n * f[j]);
                }
                if (c < D) put8<T, TAIL>((T*)p.y + row * D, c, D, v[i]);
            }
        }
        if (BLOCK && !p.u) continue;
        float sum[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[0] += (t + i * TPR) * 8 + j < D ? v[i][j] * v[i][j] : 0.0f;
        worker_sum<TPR, 1>(sum, s, turn);
        turn ^= 1;
        const float ry = 1.0f / sqrtf(sum[0] / (float)D + p.eps);
        if (p.rstd_y && t == 0) p.rstd_y[row] = ry;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int c = (t + i * TPR) * 8;
            float o[8];
            if constexpr (kLean) factors(i);
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = v[i][j] * ry * to_f32(wn[i][j]);
            if (c < D) put8<T, TAIL>((T*)p.u + row * p.ldu, c, D, o);
        }
    }
}

// Rows too wide for that: the two means of each row first, then a thread eight columns of kChunk rows.

struct Terms { float gx[8], ny[8], nh[8], f[8], g[8], s[8], w[8], gu[8]; };
template <typename T> __device__ __forceinline__ void terms8(const NormArgs& p, int64_t row, int64_t gate_row, int64_t c, float ry, float rh, float c1, Terms& t) {
    const int64_t D = p.width;
#pragma unroll
    for (int j = 0; j < 8; ++j) t.gx[j] = t.ny[j] = t.gu[j] = 0.0f;
    if (p.gy) factors8<T>((const T*)p.gy + row * D, c, D, t.gx);
    if (p.gu) {
        float wn[8];
        factors8<T>(p.wn, c, D, wn);
        factors8<T>((const T*)p.y + row * p.ldx, c, D, t.ny);
        factors8<T>((const T*)p.gu + row * p.ldg, c, D, t.gu);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            t.ny[j] *= ry;
            t.gx[j] += ry * (t.gu[j] * wn[j] - t.ny[j] * c1);
        }
    }
    if (p.h) {
        drop8(p.drop, row, c, t.f);
        factors8<T>(p.gate ? (const T*)p.gate + gate_row * D : nullptr, c, D, t.g);
        factors8<T>(p.scale, c, D, t.s);
        factors8<T>(p.w, c, D, t.w);
        factors8<T>((const T*)p.h + row * D, c, D, t.nh);
#pragma unroll
        for (int j = 0; j < 8; ++j) t.nh[j] *= rh;
    }
}

// How the backward pass divides the rows: worker k takes `rows` of them from first(k) on, all of one gate row where
// parts > 1 (that gate row's gradient is then the sum of `parts` workers'), else of whole gate rows.
struct Rows { int64_t rows, parts, workers; };

// The means of (gu w_next) n_y and of (d/dN(h)) w n_h.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_means_kernel(NormArgs p, Rows rw) {
    __shared__ float s[kThreads / 64];
    const int64_t D = p.width;
    for (int64_t row = blockIdx.x; row < p.N; row += gridDim.x) {
        const float ry = p.gu ? p.rstd_y[row] : 0.0f, rh = p.h ? p.rstd_h[row] : 0.0f;
        float c1 = 0.0f, c2 = 0.0f;
        if (p.gu) {
            for (int64_t c = threadIdx.x * 8; c < D; c += kThreads * 8) {
                float wn[8], y[8], gu[8];
                factors8<T>(p.wn, c, D, wn);
                factors8<T>((const T*)p.y + row * p.ldx, c, D, y);
                factors8<T>((const T*)p.gu + row * p.ldg, c, D, gu);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < D) c1 += gu[j] * wn[j] * (y[j] * ry);
            }
            c1 = group_sum(c1, s) / (float)D;
        }
        if (p.h) {
            for (int64_t c = threadIdx.x * 8; c < D; c += kThreads * 8) {
                Terms t;
                terms8<T>(p, row, (uint32_t)row / (uint32_t)p.rows_per_gate, c, ry, rh, c1, t);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < D && t.f[j] != 0.0f) c2 += t.gx[j] * t.s[j] * t.g[j] * t.f[j] * t.w[j] * t.nh[j];
            }
            c2 = group_sum(c2, s) / (float)D;
        }
        if (threadIdx.x == 0) {
            float* means = p.partial + (p.h && rw.parts > 1 ? rw.workers * D : 0) + rw.workers * (p.h ? 3 : 1) * D;
            means[row] = c1;
            means[p.N + row] = c2;
        }
    }
}


// A thread eight columns of one worker's rows: gx, gh, the gate's gradient and the column sums, given the means.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_columns_kernel(NormArgs p, Rows rw) {
    const int64_t D = p.width, c = ((int64_t)blockIdx.y * kThreads + threadIdx.x) * 8, worker = blockIdx.x;
    if (c >= D) return;
    int64_t r0, r1, gate_row;
    if (rw.parts > 1) {
        gate_row = worker / rw.parts;
        r0 = gate_row * p.rows_per_gate + (worker - gate_row * rw.parts) * rw.rows;
        r1 = r0 + rw.rows;
        if (r1 > (gate_row + 1) * p.rows_per_gate) r1 = (gate_row + 1) * p.rows_per_gate;
    } else {
        r0 = worker * rw.rows;
        r1 = r0 + rw.rows;
        gate_row = r0 / p.rows_per_gate;
    }
    if (r1 > p.N) r1 = p.N;
    int64_t gate_end = (gate_row + 1) * p.rows_per_gate;
    // the means of the rows lie behind the sums
    const float* means = p.partial + (p.h && rw.parts > 1 ? rw.workers * D : 0) + rw.workers * (p.h ? 3 : 1) * D;
    float sw[8] = {}, ss[8] = {}, sn[8] = {}, sg[8] = {};
    for (int64_t row = r0; row < r1; ++row) {
        const float ry = p.gu ? p.rstd_y[row] : 0.0f, rh = p.h ? p.rstd_h[row] : 0.0f;
        Terms t;
        terms8<T>(p, row, gate_row, c, ry, rh, means[row], t);
        const float c2 = means[p.N + row];
        if (p.gx) store8((T*)p.gx + row * D, c, D, t.gx);
#pragma unroll
        for (int j = 0; j < 8; ++j) sn[j] += t.gu[j] * t.ny[j];
        if (p.h) {
            float gh[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = t.f[j] == 0.0f ? 0.0f : t.gx[j] * t.f[j], m = t.f[j] == 0.0f ? 0.0f : d * t.nh[j];
                gh[j] = rh * (d * t.s[j] * t.g[j] * t.w[j] - t.nh[j] * c2);
                sw[j] += m * t.s[j] * t.g[j];
                ss[j] += m * t.w[j] * t.g[j];
                sg[j] += m * t.w[j] * t.s[j];
            }
            store8((T*)p.gh + row * D, c, D, gh);
            if (p.ggate && (row + 1 == r1 || row + 1 == gate_end)) {
                if (rw.parts > 1) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (c + j < D) p.partial[worker * D + c + j] = sg[j];
                } else {
                    store8((T*)p.ggate + gate_row * D, c, D, sg);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) sg[j] = 0.0f;
            }
        }
        if (row + 1 == gate_end) { ++gate_row; gate_end += p.rows_per_gate; }
    }
    float* out = p.partial + (p.h && rw.parts > 1 ? rw.workers * D : 0) + worker * (p.h ? 3 : 1) * D + c;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (c + j < D) {
            if (p.h) {
                out[j] = sw[j];
                out[D + j] = ss[j];
                out[2 * D + j] = sn[j];
            } else {
                out[j] = sn[j];
            }
        }
}

// One pass over the rows: gx, gh, the gate's gradient, and each work-group's column sums (of w, scale, w_next).
// With q = scale gate drop w n_h, the two means of a row need three sums and no second pass:
//   c1 = mean(gu w_next n_y),  c2 = mean((gy + r_y gu w_next) q) - r_y c1 mean(n_y q)
template <typename T, int TPR, int I, bool TAIL, bool H>
__global__ __launch_bounds__(group_of(TPR)) void norm_backward_rows(NormArgs p, Rows rw) {
    constexpr int kGroup = group_of(TPR), kWorkers = kGroup / TPR, kSums = H ? 3 : 1, B = H ? I : 1;
    __shared__ float s[2 * 3 * (TPR > 64 ? TPR / 64 : 1)];
    __shared__ float cols[kWorkers > 1 ? kWorkers * TPR * I * 8 : 1];
    typedef typename Raw<T>::V V;
    const int D = (int)p.width, t = threadIdx.x % TPR;
    const int64_t worker = (int64_t)blockIdx.x * kWorkers + threadIdx.x / TPR;
    int64_t r0, r1, gate_row = 0;
    if (rw.parts > 1) {
        gate_row = worker / rw.parts;
        r0 = gate_row * p.rows_per_gate + (worker - gate_row * rw.parts) * rw.rows;
        r1 = r0 + rw.rows;
        if (r1 > (gate_row + 1) * p.rows_per_gate) r1 = (gate_row + 1) * p.rows_per_gate;
    } else {
        r0 = worker * rw.rows;
        r1 = r0 + rw.rows;
        gate_row = r0 / p.rows_per_gate;
    }
    if (r1 > p.N) r1 = p.N;
    if (worker >= rw.workers) r1 = r0;
    int64_t gate_end = (gate_row + 1) * p.rows_per_gate;

    float sw[B][8] = {}, ss[B][8] = {}, sg[B][8] = {}, sn[I][8] = {};
    V gyr[I], gur[I], yr[I], hr[B], gr[B], wn[I], w[B], sc[B];
    float ryr = 0.0f, rhr = 0.0f;
#pragma unroll
    for (int i = 0; i < I; ++i) gyr[i] = gur[i] = yr[i] = V{};
    auto fetch = [&](int64_t row) {
        const T* gate = H && p.gate ? (const T*)p.gate + gate_row * D : nullptr;
        if (p.gu) ryr = p.rstd_y[row];
        if constexpr (H) rhr = p.rstd_h[row];
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int c = (t + i * TPR) * 8;
            if (p.gy) gyr[i] = row8<T, TAIL>((const T*)p.gy + row * D, c, D);
            if (p.gu) {
                gur[i] = row8<T, TAIL>((const T*)p.gu + row * p.ldg, c, D);
                yr[i] = row8<T, TAIL>((const T*)p.y + row * p.ldx, c, D);
            }
            if constexpr (H) {
                hr[i] = row8<T, TAIL>((const T*)p.h + row * D, c, D);
                gr[i] = ones8<T, TAIL>(gate, c, D);
            }
        }
    };
    constexpr bool kLean = TPR == 1024;
    if (!kLean && r0 < r1) fetch(r0);
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int c = (t + i * TPR) * 8;
        if constexpr (!kLean) wn[i] = ones8<T, TAIL>(p.wn, c, D);
        if constexpr (H) {
            w[i] = ones8<T, TAIL>(p.w, c, D);
            sc[i] = ones8<T, TAIL>(p.scale, c, D);
        }
    }
    int turn = 0;
    for (int64_t row = r0; row < r1; ++row, turn ^= 1) {
        if constexpr (kLean) fetch(row);
        // per value: a = gy + r_y gu w_next, n_y, and for the block's side n_h and the dropout's factor
        const float ry = ryr, rh = rhr;
        float a[I][8], ny[I][8], nh[B][8], f[B][8];
        V g[B];
        float sum[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int c = (t + i * TPR) * 8;
            if constexpr (kLean) wn[i] = ones8<T, TAIL>(p.wn, c, D);
            if constexpr (H) {
                g[i] = gr[i];
                drop8(p.drop, row, c, f[i]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float gu = to_f32(gur[i][j]), gw = gu * to_f32(wn[i][j]);
                ny[i][j] = to_f32(yr[i][j]) * ry;
                sum[0] += gw * ny[i][j];
                sn[i][j] += gu * ny[i][j];
                a[i][j] = to_f32(gyr[i][j]) + ry * gw;
                if constexpr (H) {
                    nh[i][j] = to_f32(hr[i][j]) * rh;
                    const float q = f[i][j] == 0.0f ? 0.0f : to_f32(sc[i][j]) * to_f32(g[i][j]) * f[i][j] * to_f32(w[i][j]) * nh[i][j];
                    sum[1] += a[i][j] * q;
                    sum[2] += ny[i][j] * q;
                }
            }
        }
        const bool last = row + 1 == r1 || row + 1 == gate_end;   // of this gate row, or of this worker
        const int64_t gate_at = gate_row;
        if (row + 1 < r1) {
            if (row + 1 == gate_end) { ++gate_row; gate_end += p.rows_per_gate; }
            if constexpr (!kLean) fetch(row + 1);
        }
        if constexpr (H) {
            worker_sum<TPR, 3>(sum, s, turn);
        } else {
            float one[1] = {sum[0]};
            worker_sum<TPR, 1>(one, s, turn);
            sum[0] = one[0];
        }
        const float c1 = sum[0] / (float)D, c2 = (sum[1] - ry * c1 * sum[2]) / (float)D;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int c = (t + i * TPR) * 8;
            if (c >= D) continue;
            float gx[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) gx[j] = a[i][j] - ry * ny[i][j] * c1;
            if (p.gx) put8<T, TAIL>((T*)p.gx + row * D, c, D, gx);
            if constexpr (H) {
                float gh[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float wj = to_f32(w[i][j]), gj = to_f32(g[i][j]), sj = to_f32(sc[i][j]);
                    const float d = f[i][j] == 0.0f ? 0.0f : gx[j] * f[i][j];     // with respect to scale gate N(h)
                    const float m = f[i][j] == 0.0f ? 0.0f : d * nh[i][j];
                    const float gv = d * sj * gj;
                    gh[j] = rh * (gv * wj - nh[i][j] * c2);
                    sw[i][j] += m * sj * gj;
                    ss[i][j] += m * wj * gj;
                    sg[i][j] += m * wj * sj;
                }
                put8<T, TAIL>((T*)p.gh + row * D, c, D, gh);
                if (p.ggate && last) {
                    if (rw.parts > 1) {
                        float* to = p.partial + worker * D;   // gate rows' parts come first
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (c + j < D) to[c + j] = sg[i][j];
                    } else {
                        put8<T, TAIL>((T*)p.ggate + gate_at * D, c, D, sg[i]);
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) sg[i][j] = 0.0f;
                }
            }
        }
    }

    // column sums of the work-group
    const int64_t gates_at = H && rw.parts > 1 ? rw.workers * D : 0;
    float* out = p.partial + gates_at + (int64_t)blockIdx.x * kSums * D;
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        if constexpr (kWorkers > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    cols[(threadIdx.x / TPR) * (TPR * I * 8) + (t + i * TPR) * 8 + j] = k == kSums - 1 ? sn[i][j] : k == 0 ? sw[H ? i : 0][j] : ss[H ? i : 0][j];
            __syncthreads();
            for (int c = threadIdx.x; c < D; c += kGroup) {
                float v = 0.0f;
#pragma unroll
                for (int w = 0; w < kWorkers; ++w) v += cols[w * (TPR * I * 8) + c];
                out[(int64_t)k * D + c] = v;
            }
        } else {
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const int c = (t + i * TPR) * 8;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < D) out[(int64_t)k * D + c + j] = k == kSums - 1 ? sn[i][j] : k == 0 ? sw[H ? i : 0][j] : ss[H ? i : 0][j];
            }
        }
    }
}

// The work-groups' column sums added up, 64 columns a work-group, sixteen strands of rows; then, by the work-groups
// after those, the parts of each gate row.  Every sum is taken in a fixed order.
template <typename T>
__global__ __launch_bounds__(1024) void norm_join_kernel(NormArgs p, Rows rw, int64_t groups, int sums) {
    const int64_t D = p.width, blocks = (D + 63) / 64, c = (int64_t)(blockIdx.x % blocks) * 64 + (threadIdx.x & 63);
    const int strand = threadIdx.x >> 6;
    const int64_t job = blockIdx.x / blocks;
    const bool gates = job >= sums;
    const float* from;
    int64_t n;
    const bool split = sums == 3 && rw.parts > 1;
    if (gates) {
        const int64_t gate = job - sums;
        from = p.partial + gate * rw.parts * D + c;
        // the last gate row may have fewer rows: the workers beyond them wrote nothing
        const int64_t left = (p.N - gate * p.rows_per_gate + rw.rows - 1) / rw.rows;
        n = left < rw.parts ? left : rw.parts;
    } else {
        from = p.partial + (split ? rw.workers * D : 0) + job * D + c;
        n = groups;
    }
    const int64_t step = gates ? D : sums * D;
    float v = 0.0f, u[8] = {};
    if (c < D) {
        int64_t i = strand;
        for (; i + 112 < n; i += 128)   // eight loads in flight
#pragma unroll
            for (int k = 0; k < 8; ++k) u[k] += from[(i + 16 * k) * step];
        for (; i < n; i += 16) v += from[i * step];
#pragma unroll
        for (int k = 0; k < 8; ++k) v += u[k];
    }
    __shared__ float s[16][64];
    s[strand][threadIdx.x & 63] = v;
    __syncthreads();
    if (strand || c >= D) return;
#pragma unroll
    for (int k = 1; k < 16; ++k) v += s[k][threadIdx.x];
    if (gates) {
        ((T*)p.ggate)[(job - sums) * D + c] = (T)v;
    } else {
        void* to = job == sums - 1 ? p.gwn : job == 0 ? p.gw : p.gscale;
        if (to) ((T*)to)[c] = (T)v;
    }
}

// Threads a row and turns for a width; none below a chunk and above what registers hold.  The backward pass of a block's side carries
// four column sums and ten values a column and takes one turn (190 registers); the others take two.
enum Pass { kForward, kBackward, kBackwardBlock };
struct Shape { int tpr, turns; };
inline Shape shape_of(int64_t width, Pass pass) {
    const int64_t chunks = (width + 7) / 8;
    if (width < 8) return {0, 0};   // row8 reads eight values
    for (int t : {8, 16, 32, 64})
        if (chunks <= t) return {t, 1};
    if (pass == kBackwardBlock) {
        for (int t : {128, 256, 512})
            if (chunks <= t) return {t, 1};
        return {0, 0};
    }
    if (chunks <= 128) return {64, 2};
    if (pass == kForward && chunks <= 192) return {192, 1};   // (the backward pass: 54 us a pass of 4001 x 1089, 38 with 256)
    if (chunks <= 256) return {256, 1};
    for (int t : {256, 512, 1024})
        if (chunks <= 2 * t) return {t, 2};
    return {0, 0};
}

// Workers of the column kernel: about four work-groups a compute unit over all columns.
inline int64_t column_blocks(int64_t width) { return (width + 8 * kThreads - 1) / (8 * kThreads); }

inline Rows rows_of(const Shape& sh, int64_t width, int64_t N, int64_t rows_per_gate) {
    // eight waves a compute unit
    const int64_t wide = 1024 / column_blocks(width), want = sh.tpr ? 512 * 256 / sh.tpr : wide > 1 ? wide : 1;
    int64_t r = (N + want - 1) / want;
    if (r < 4) r = 4;
    Rows out;
    if (rows_per_gate > r) {
        out.parts = (rows_per_gate + r - 1) / r;
        out.rows = (rows_per_gate + out.parts - 1) / out.parts;
        out.workers = (N + rows_per_gate - 1) / rows_per_gate * out.parts;
    } else {
        out.parts = 1;
        out.rows = r / rows_per_gate * rows_per_gate;
        out.workers = (N + out.rows - 1) / out.rows;
    }
    return out;
}

inline int64_t groups_for(const Rows& r, const Shape& sh) {
    const int64_t per = sh.tpr ? group_of(sh.tpr) / sh.tpr : 1;
    return (r.workers + per - 1) / per;
}

// A thread a block of eight columns (one call of the generator) and turn; the row and block of its next turn follow
// from the last one's without a division.
template <typename T>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const T* x, int64_t ldx, T* y, int64_t ldy, int64_t N, int64_t width,
                                                           DropArgs d, int64_t step_rows, int64_t step_blocks) {
    const int64_t blocks = (width + 7) / 8;
    const int64_t first = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    int64_t row = first / blocks, b = first - row * blocks;
    while (row < N) {
        const typename Raw<T>::V v = load8(x + row * ldx, b * 8, width);
        const Words q = philox((uint32_t)b, (uint32_t)row, d.offset, d.seed);
        float o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = kept(q, j, d.threshold) ? to_f32(v[j]) * d.scale : 0.0f;
        store8(y + row * ldy, b * 8, width, o);
        row += step_rows;
        b += step_blocks;
        if (b >= blocks) { b -= blocks; ++row; }
    }
}

inline unsigned row_groups(int64_t N) { return (unsigned)(N < (1 << 20) ? N : 1 << 20); }

#define FFN_SHAPES(RUN)                                  \
    switch (sh.tpr * 8 + sh.turns) {                     \
        case 8 * 8 + 1: RUN(8, 1); break;                \
        case 16 * 8 + 1: RUN(16, 1); break;              \
        case 32 * 8 + 1: RUN(32, 1); break;              \
        case 64 * 8 + 1: RUN(64, 1); break;              \
        case 64 * 8 + 2: RUN(64, 2); break;              \
        case 192 * 8 + 1: RUN(192, 1); break;            \
        case 256 * 8 + 1: RUN(256, 1); break;            \
        case 256 * 8 + 2: RUN(256, 2); break;            \
        case 512 * 8 + 2: RUN(512, 2); break;            \
        default: RUN(1024, 2); break;                    \
    }

template <typename T> int forward(const NormArgs& a, hipStream_t s) {
    const Shape sh = shape_of(a.width, kForward);
    if (sh.tpr == 0) {
        norm_forward_kernel<T><<<dim3(row_groups(a.N)), kThreads, 0, s>>>(a);
        return (int)hipGetLastError();
    }
    const bool tail = a.width % 8 != 0, block = a.h != nullptr;
    // up to sixteen waves a compute unit walk the rows
    const int64_t per = group_of(sh.tpr) / sh.tpr, all = (a.N + per - 1) / per, most = 256 * 1024 / group_of(sh.tpr);
    const dim3 grid((unsigned)(all < most ? all : most));
#define FFN_FORWARD(TPR, I)                                                                              \
    if (block && tail) norm_forward_rows<T, TPR, I, true, true><<<grid, group_of(TPR), 0, s>>>(a);      \
    else if (block) norm_forward_rows<T, TPR, I, false, true><<<grid, group_of(TPR), 0, s>>>(a);        \
    else if (tail) norm_forward_rows<T, TPR, I, true, false><<<grid, group_of(TPR), 0, s>>>(a);         \
    else norm_forward_rows<T, TPR, I, false, false><<<grid, group_of(TPR), 0, s>>>(a)
    FFN_SHAPES(FFN_FORWARD)
#undef FFN_FORWARD
    return (int)hipGetLastError();
}

template <typename T> int backward(const NormArgs& a, hipStream_t s) {
    const bool block = a.h != nullptr, tail = a.width % 8 != 0;
    const Shape sh = shape_of(a.width, block ? kBackwardBlock : kBackward);
    const Rows rw = rows_of(sh, a.width, a.N, block ? a.rows_per_gate : 1);
    const int64_t groups = groups_for(rw, sh);
    if (sh.tpr == 0 && groups > 0) {
        norm_means_kernel<T><<<dim3(row_groups(a.N)), kThreads, 0, s>>>(a, rw);
        norm_columns_kernel<T><<<dim3((unsigned)groups, (unsigned)column_blocks(a.width)), kThreads, 0, s>>>(a, rw);
    } else if (groups > 0 && block) {
#define FFN_BLOCK(TPR)                                                                                              \
    if (tail) norm_backward_rows<T, TPR, 1, true, true><<<dim3((unsigned)groups), group_of(TPR), 0, s>>>(a, rw);    \
    else norm_backward_rows<T, TPR, 1, false, true><<<dim3((unsigned)groups), group_of(TPR), 0, s>>>(a, rw)
        switch (sh.tpr) {
            case 8: FFN_BLOCK(8); break;
            case 16: FFN_BLOCK(16); break;
            case 32: FFN_BLOCK(32); break;
            case 64: FFN_BLOCK(64); break;
            case 128: FFN_BLOCK(128); break;
            case 256: FFN_BLOCK(256); break;
            default: FFN_BLOCK(512); break;
        }
#undef FFN_BLOCK
    } else if (groups > 0) {
#define FFN_BACKWARD(TPR, I)                                                                                        \
    if (tail) norm_backward_rows<T, TPR, I, true, false><<<dim3((unsigned)groups), group_of(TPR), 0, s>>>(a, rw);   \
    else norm_backward_rows<T, TPR, I, false, false><<<dim3((unsigned)groups), group_of(TPR), 0, s>>>(a, rw)
        FFN_SHAPES(FFN_BACKWARD)
#undef FFN_BACKWARD
    }
    if (a.gw || a.gscale || a.gwn || (a.ggate && rw.parts > 1)) {
        const int sums = block ? 3 : 1;
        const int64_t jobs = sums + (a.ggate && rw.parts > 1 ? (a.N + a.rows_per_gate - 1) / a.rows_per_gate : 0);
        norm_join_kernel<T><<<dim3((unsigned)(jobs * ((a.width + 63) / 64))), 1024, 0, s>>>(a, rw, groups, sums);
    }
    return (int)hipGetLastError();
}

template <typename T> int drop(const void* x, int64_t ldx, void* y, int64_t ldy, int64_t N, int64_t width, const DropArgs& d, hipStream_t s) {
    const int64_t blocks = (width + 7) / 8, groups = (N * blocks + kThreads - 1) / kThreads;
    const dim3 grid((unsigned)(groups < 4096 ? groups : 4096));
    const int64_t stride = (int64_t)grid.x * kThreads, dr = stride / blocks, db = stride % blocks;
    dropout_kernel<T><<<grid, kThreads, 0, s>>>((const T*)x, ldx, (T*)y, ldy, N, width, d, dr, db);
    return (int)hipGetLastError();
}

inline int64_t workspace_floats(int64_t width, int64_t N, int64_t rows_per_gate, bool residual) {
    const Shape sh = shape_of(width, residual ? kBackwardBlock : kBackward);
    const Rows rw = rows_of(sh, width, N, residual ? rows_per_gate : 1);
    return (residual && rw.parts > 1 ? rw.workers * width : 0) + groups_for(rw, sh) * (residual ? 3 : 1) * width + (sh.tpr ? 0 : 2 * N);
}

}  // namespace
}  // namespace ffn
