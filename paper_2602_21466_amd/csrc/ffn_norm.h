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

// One row a work-group, eight columns a thread and turn: rows too narrow or too wide for registers.  y = x + scale * gate *
// drop(N(h; w)) where h is given, then u = N(y; wn).  A row is read again for each sum, from the caches while it fits them
// (1000 x 40000 in bf16: 55 us, 151 with the block's side;
// by single values 184 and 643).
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_forward_kernel(NormArgs p) {
    __shared__ float s[kThreads / 64];
    const int64_t D = p.width;
    for (int64_t row = blockIdx.x; row < p.N; row += gridDim.x) {
        const T* x = (const T*)p.x + row * p.ldx;
        const T* h = p.h ? (const T*)p.h + row * D : nullptr;
        const T* gate = p.h && p.gate ? (const T*)p.gate + row / p.rows_per_gate * D : nullptr;
        float rh = 0.0f;
        if (h) {
            float sum = 0.0f;
            for (int64_t c = threadIdx.x * 8; c < D; c += kThreads * 8) {
                float v[8];
                factors8<T>(h, c, D, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum += v[j] * v[j];   // (zeros beyond the row)
            }
            rh = 1.0f / sqrtf(group_sum(sum, s) / (float)D + p.eps);
            if (p.rstd_h && threadIdx.x == 0) p.rstd_h[row] = rh;
        }
        auto joined = [&](int64_t c, float (&v)[8]) {
            factors8<T>(x, c, D, v);
            if (!h) return;
            float n[8], w[8], sc[8], g[8], f[8];
            factors8<T>(h, c, D, n);
            factors8<T>(p.w, c, D, w);
            factors8<T>(p.scale, c, D, sc);
            factors8<T>(gate, c, D, g);
            drop8(p.drop, row, c, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += sc[j] * g[j] * (f[j] == 0.0f ? 0.0f : n[j] * rh * w[j] * f[j]);
        };
        float sum = 0.0f;
        for (int64_t c = threadIdx.x * 8; c < D; c += kThreads * 8) {
            float v[8];
            joined(c, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += c + j < D ? v[j] * v[j] : 0.0f;
            if (!p.u) store8((T*)p.y + row * D, c, D, v);
        }
        if (!p.u) continue;
        const float ry = 1.0f / sqrtf(group_sum(sum, s) / (float)D + p.eps);
        if (p.rstd_y && threadIdx.x == 0) p.rstd_y[row] = ry;
        for (int64_t c = threadIdx.x * 8; c < D; c += kThreads * 8) {
            float v[8], wn[8];
            joined(c, v);
            if (p.y) store8((T*)p.y + row * D, c, D, v);
            factors8<T>(p.wn, c, D, wn);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= ry * wn[j];
            store8((T*)p.u + row * p.ldu, c, D, v);
        }
    }
}

// The kept of the generator's block of eight columns, bit j for column j; and of a row's columns c .. c + 7.
__device__ __forceinline__ uint32_t block_mask(const DropArgs& d, int64_t row, int block) {
    const Words q = philox((uint32_t)block, (uint32_t)row, d.offset, d.seed);
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m |= kept(q, j, d.threshold) ? 1u << j : 0u;
    return m;
}
template <bool TAIL> __device__ __forceinline__ uint32_t mask8(const DropArgs& d, int64_t row, int c) {
    if (d.threshold == 0) return 0xFFu;
    if constexpr (!TAIL) return block_mask(d, row, c >> 3);
    uint32_t m = 0;
#pragma unroll 1
    for (int b = (c + 7) >> 3; b >= c >> 3; --b) m = m << 8 | block_mask(d, row, b);   // two where c is inside a block
    return m >> (c & 7);
}

template <int CONTROL> __device__ __forceinline__ float moved(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CONTROL, 0xF, 0xF, true));
}
__device__ __forceinline__ float lane(float v, int l) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l));
}

// Sums of K values over a worker, returned to all its threads.  `s` is LDS for two calls in turn (`turn` alternates):
// one barrier a call keeps both the values and the next but one call's writes in order.
template <int TPR, int K> __device__ __forceinline__ void worker_sum(float (&v)[K], float* s, int turn) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
        v[k] += moved<0xB1>(v[k]);                                    // lane ^ 1
        v[k] += moved<0x4E>(v[k]);                                    // lane ^ 2
        v[k] += moved<0x141>(v[k]);                                   // the other four of eight, mirrored
        if constexpr (TPR >= 16) v[k] += moved<0x140>(v[k]);          // the other eight of sixteen, mirrored
        if constexpr (TPR == 32) v[k] += __shfl_xor(v[k], 16, 64);
        if constexpr (TPR >= 64) v[k] = (lane(v[k], 0) + lane(v[k], 16)) + (lane(v[k], 32) + lane(v[k], 48));
    }
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

// Eight values as they were loaded, in words: a vector of 16-bit values that lives across a loop takes a register each.
template <typename T> struct Eight {
    static constexpr int W = 2 * sizeof(T);
    uint32_t w[W];
};
template <typename T> __device__ __forceinline__ float at(const Eight<T>& v, int j) {
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(float, v.w[j]);
    } else {
        typedef T P __attribute__((ext_vector_type(2)));
        return to_f32(__builtin_bit_cast(P, v.w[j / 2])[j & 1]);
    }
}

// Hides where the words came from, so that what was computed from them is computed again and not held.
template <typename T> __device__ __forceinline__ void keep(Eight<T>& v) {
#pragma unroll
    for (int k = 0; k < Eight<T>::W; ++k) asm volatile("" : "+v"(v.w[k]));
}

// The eight columns of a row of D >= 8 that a thread takes in a turn: from c on, the first `skip` of them another
// thread's as well (all eight where the thread has none).  TAIL: D is no multiple of 8, and the last thread takes the
// row's last eight columns: it writes what its neighbour writes where they overlap and leaves those out of the row's sums.
// (4001 x 1089 in fp16, the gradients: 23 us; 32 to 37 with loads moved into place and stores by fewer values there.)
struct Place { int c, skip; };
template <bool TAIL> __device__ __forceinline__ Place place8(int c, int D) {
    Place p = {c, c < D ? 0 : 8};
    if (TAIL && c < D && c > D - 8) p = {D - 8, c - (D - 8)};
    return p;
}
template <typename T> __device__ __forceinline__ Eight<T> row8(const T* row, const Place& p) {
    Eight<T> v = {};
    if (p.skip < 8) __builtin_memcpy(&v, (const char*)row + (uint32_t)p.c * (uint32_t)sizeof(T), sizeof(v));
    return v;
}
template <typename T> __device__ __forceinline__ void put8(T* row, const Place& p, const float (&f)[8]) {
    typename Raw<T>::V v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (T)f[j];
    __builtin_memcpy((char*)row + (uint32_t)p.c * (uint32_t)sizeof(T), &v, sizeof(v));
}
// A row of factors, ones where there is none.
template <typename T> __device__ __forceinline__ Eight<T> ones8(const void* p, const Place& at) {
    if (p) return row8<T>((const T*)p, at);
    Eight<T> v;
    T one[4 / sizeof(T)];
    for (T& o : one) o = (T)1.0f;
#pragma unroll
    for (int k = 0; k < Eight<T>::W; ++k) __builtin_memcpy(&v.w[k], one, 4);
    return v;
}

constexpr int group_of(int tpr) { return tpr > 64 ? tpr : 256; }
// Waves a SIMD that the backward rows' registers are bounded for (128 registers hold four, 168 three), and that are
// started.  Rows of a wave or more have scalar addresses.
constexpr int backward_waves(int bytes, int tpr, int turns, bool block) {
    if (!block) return turns == 1 || tpr == 1024 ? 4 : 3;
    if (turns == 2) return 2;
    return bytes == 2 ? tpr >= 64 ? 4 : 3 : tpr >= 64 && tpr < 512 ? 3 : 2;
}

constexpr int forward_waves(int bytes, int tpr, int turns, bool block) {
    if (tpr == 1024 || !block) return 4;   // (eight: 6.7 us, not 6.4, at 8192 x 289)
    return turns == 2 ? bytes == 2 ? 4 : 3 : bytes == 2 ? 6 : 4;
}

// BLOCK: y = x + scale gate drop(N(h; w)) first.  A worker walks its rows with the next one's loads in flight, the
// factors shared by all rows in registers; workers of 1024 threads have 128 registers each and do neither.  Bound by HBM:
// 5.2 TB/s at 16384 x 4096 in bf16 (104 us, the block's side and the next norm).
template <typename T, int TPR, int I, bool TAIL, bool BLOCK>
__global__ __launch_bounds__(group_of(TPR), forward_waves(sizeof(T), TPR, I, BLOCK)) void norm_forward_rows(NormArgs p) {
    __shared__ float s[2 * (TPR > 64 ? TPR / 64 : 1)];
    constexpr int kWorkers = group_of(TPR) / TPR, B = BLOCK ? I : 1;
    typedef Eight<T> V;
    const int D = (int)p.width, t = threadIdx.x % TPR;
    const int64_t step = (int64_t)gridDim.x * kWorkers;
    const int sub = kWorkers == 1 ? 0 : TPR < 64 ? threadIdx.x / TPR : __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    int64_t row = (int64_t)blockIdx.x * kWorkers + sub;
    if (row >= p.N) return;
    V wn[I], w[B], sc[B], xr[I], hr[B], gr[B];
    Place at8[I];
#pragma unroll
    for (int i = 0; i < I; ++i) at8[i] = place8<TAIL>((t + i * TPR) * 8, D);
    auto fetch = [&](int64_t r) {
        const T* gate = BLOCK && p.gate ? (const T*)p.gate + (int64_t)((uint32_t)r / (uint32_t)p.rows_per_gate) * D : nullptr;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            xr[i] = row8<T>((const T*)p.x + r * p.ldx, at8[i]);
            if constexpr (BLOCK) {
                hr[i] = row8<T>((const T*)p.h + r * D, at8[i]);
                gr[i] = ones8<T>(gate, at8[i]);
            }
        }
    };
    constexpr bool kLean = TPR == 1024;
    auto factors = [&](int i) {
        wn[i] = ones8<T>(p.wn, at8[i]);
        if constexpr (BLOCK) {
            w[i] = ones8<T>(p.w, at8[i]);
            sc[i] = ones8<T>(p.scale, at8[i]);
        }
    };
    if constexpr (!kLean) {
        fetch(row);
#pragma unroll
        for (int i = 0; i < I; ++i) factors(i);
    }
    for (int turn = 0; row < p.N; row += step) {
#pragma unroll
        for (int i = 0; i < I; ++i) {   // neither lanes' addresses nor converted factors are held over the rows
            if constexpr (!kLean) {
                asm volatile("" : "+v"(at8[i].c));
                keep(wn[i]);
                if constexpr (BLOCK) {
                    keep(w[i]);
                    keep(sc[i]);
                }
            }
        }
        if constexpr (kLean) fetch(row);
        float v[I][8];
        V h[B], g[B];
#pragma unroll
        for (int i = 0; i < I; ++i) {
            if constexpr (TAIL && BLOCK) keep(xr[i]);   // here before another thread may write y over it
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = at(xr[i], j);
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
                for (int j = 0; j < 8; ++j) sum[0] += !TAIL || j >= at8[i].skip ? at(h[i], j) * at(h[i], j) : 0.0f;
            worker_sum<TPR, 1>(sum, s, turn);
            turn ^= 1;
            const float fs = p.drop.threshold ? p.drop.scale : 1.0f;
            const float rh = 1.0f / sqrtf(sum[0] / (float)D + p.eps);
            if (p.rstd_h && t == 0) p.rstd_h[row] = rh;
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const uint32_t mask = mask8<TAIL>(p.drop, row, at8[i].c);
                if constexpr (kLean) factors(i);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float n = at(h[i], j) * rh * at(w[i], j);
                    v[i][j] += at(sc[i], j) * at(g[i], j) * (mask >> j & 1 ? n * fs : 0.0f);
                }
                if (at8[i].skip < 8) put8<T>((T*)p.y + row * D, at8[i], v[i]);
            }
        }
        if (BLOCK && !p.u) continue;
        float sum[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[0] += (TAIL ? j >= at8[i].skip : at8[i].skip == 0) ? v[i][j] * v[i][j] : 0.0f;
        worker_sum<TPR, 1>(sum, s, turn);
        turn ^= 1;
        const float ry = 1.0f / sqrtf(sum[0] / (float)D + p.eps);
        if (p.rstd_y && t == 0) p.rstd_y[row] = ry;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            float o[8];
            if constexpr (kLean) factors(i);
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = v[i][j] * ry * at(wn[i], j);
            if (at8[i].skip < 8) put8<T>((T*)p.u + row * p.ldu, at8[i], o);
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

// How the backward pass divides the rows.  parts > 1: worker k takes the rows k mod parts, + parts, .. of gate row k / parts,
// whose gradient is then the sum of `parts` workers'.  Else it takes the gate rows k, k + workers, .., each whole.  Either way
// rows read at one time lie side by side.
struct Rows { int64_t parts, workers; };
struct Walk {
    int64_t row, gate_row, gate_end;
    __device__ Walk(const NormArgs& p, const Rows& rw, int64_t worker) {
        gate_row = rw.parts > 1 ? worker / rw.parts : worker;
        row = gate_row * p.rows_per_gate + (rw.parts > 1 ? worker - gate_row * rw.parts : 0);
        if (worker >= rw.workers) row = p.N;
        limit(p);
    }
    __device__ void limit(const NormArgs& p) {
        gate_end = (gate_row + 1) * p.rows_per_gate;
        if (gate_end > p.N) gate_end = p.N;
    }
    // Whether this worker has no row of this gate row after this one.
    __device__ bool last(const Rows& rw) const { return row + rw.parts >= gate_end; }
    __device__ void advance(const NormArgs& p, const Rows& rw) {
        row += rw.parts;
        if (row < gate_end) return;
        if (rw.parts > 1) {
            row = p.N;
        } else {
            gate_row += rw.workers;
            row = gate_row * p.rows_per_gate;
            limit(p);
        }
    }
};

// The means of (gu w_next) n_y and of (d/dN(h)) w n_h, a row a work-group: all arrays are read here and again by the
// columns' kernel (4000 x 12000 in bf16: 136 us and 254, 3.5 and 3.2 TB/s; rows of fewer than eight columns leave most of
// a work-group idle, 100000 x 4 in fp32: 175 us and 180).
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
            float* means = p.partial + (p.h && rw.parts > 1 ? rw.workers * D : 0) + rw.workers * (p.h ? 2 : 1) * D;
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
    // the means of the rows lie behind the sums
    const float* means = p.partial + (p.h && rw.parts > 1 ? rw.workers * D : 0) + rw.workers * (p.h ? 2 : 1) * D;
    float sm[8] = {}, sn[8] = {}, sg[8] = {};
    for (Walk k(p, rw, worker); k.row < p.N; k.advance(p, rw)) {
        const int64_t row = k.row;
        const float ry = p.gu ? p.rstd_y[row] : 0.0f, rh = p.h ? p.rstd_h[row] : 0.0f;
        Terms t;
        terms8<T>(p, row, k.gate_row, c, ry, rh, means[row], t);
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
                sm[j] += m * t.g[j];
                sg[j] += m * t.w[j] * t.s[j];
            }
            store8((T*)p.gh + row * D, c, D, gh);
            if (p.ggate && k.last(rw)) {
                if (rw.parts > 1) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (c + j < D) p.partial[worker * D + c + j] = sg[j];
                } else {
                    store8((T*)p.ggate + k.gate_row * D, c, D, sg);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) sg[j] = 0.0f;
            }
        }
    }
    float* out = p.partial + (p.h && rw.parts > 1 ? rw.workers * D : 0) + worker * (p.h ? 2 : 1) * D + c;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (c + j < D) {
            if (p.h) {
                out[j] = sm[j];
                out[D + j] = sn[j];
            } else {
                out[j] = sn[j];
            }
        }
}

// One pass over the rows: gx, gh, the gate's gradient, and each work-group's column sums.
// With q = scale gate drop w n_h, the two means of a row need three sums and no second pass:
//   c1 = mean(gu w_next n_y),  c2 = mean((gy + r_y gu w_next) q) - r_y c1 mean(n_y q)
// and with m = (d/dN(h)) / (scale gate w) n_h one sum a gate row, M = sum m, serves three gradients:
//   d gate = scale w M,  d w = scale sum(gate M),  d scale = w sum(gate M)   (the factors over columns by the joining kernel).
// Bound by HBM: 4.8 TB/s at 16384 x 4096 in bf16 (174 us).  The registers decide how many waves hide the loads: between the
// two halves of a row's work its arrays stay as they were loaded, and what follows from them is computed again (126 registers
// for 16-bit arrays, four waves a SIMD; with the computed values held it took 190, two waves and 37 us where it now takes 23,
// at 4001 x 1089 in fp16).
template <typename T, int TPR, int I, bool TAIL, bool H>
__global__ __launch_bounds__(group_of(TPR), backward_waves(sizeof(T), TPR, I, H)) void norm_backward_rows(NormArgs p, Rows rw) {
    constexpr int kGroup = group_of(TPR), kWorkers = kGroup / TPR, kSums = H ? 2 : 1, B = H ? I : 1;
    __shared__ float s[2 * 3 * (TPR > 64 ? TPR / 64 : 1)];
    __shared__ float cols[kWorkers > 1 ? kWorkers * TPR * I * 8 : 1];
    typedef Eight<T> V;
    const int D = (int)p.width, t = threadIdx.x % TPR;
    const int sub = kWorkers == 1 ? 0 : TPR < 64 ? threadIdx.x / TPR : __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    const int64_t worker = (int64_t)blockIdx.x * kWorkers + sub;
    Walk k(p, rw, worker);

    float sm[B][8] = {}, sg[B][8] = {}, sn[I][8] = {};   // M, sum(gate M), and w_next's
    V gyr[I], gur[I], yr[I], hr[B], gr[B], wn[I], w[B], sc[B];
    float ryr = 0.0f, rhr = 0.0f;
    Place at8[I];
#pragma unroll
    for (int i = 0; i < I; ++i) at8[i] = place8<TAIL>((t + i * TPR) * 8, D);
#pragma unroll
    for (int i = 0; i < I; ++i) gyr[i] = gur[i] = yr[i] = V{};
    auto fetch = [&](int64_t row, int64_t gate_row) {
        const T* gate = H && p.gate ? (const T*)p.gate + gate_row * D : nullptr;
        if (p.gu) ryr = p.rstd_y[row];
        if constexpr (H) rhr = p.rstd_h[row];
#pragma unroll
        for (int i = 0; i < I; ++i) {
            if (p.gy) gyr[i] = row8<T>((const T*)p.gy + row * D, at8[i]);
            if (p.gu) {
                gur[i] = row8<T>((const T*)p.gu + row * p.ldg, at8[i]);
                yr[i] = row8<T>((const T*)p.y + row * p.ldx, at8[i]);
            }
            if constexpr (H) {
                hr[i] = row8<T>((const T*)p.h + row * D, at8[i]);
                gr[i] = ones8<T>(gate, at8[i]);
            }
        }
    };
    constexpr bool kLean = TPR == 1024;
    if (!kLean && k.row < p.N) fetch(k.row, k.gate_row);
#pragma unroll
    for (int i = 0; i < I; ++i) {
        if constexpr (!kLean) wn[i] = ones8<T>(p.wn, at8[i]);
        if constexpr (H) {
            w[i] = ones8<T>(p.w, at8[i]);
            sc[i] = ones8<T>(p.scale, at8[i]);
        }
    }
    for (int turn = 0; k.row < p.N; turn ^= 1) {
        const int64_t row = k.row, gate_row = k.gate_row;
#pragma unroll
        for (int i = 0; i < I; ++i) {   // neither lanes' addresses nor converted factors are held over the rows
            asm volatile("" : "+v"(at8[i].c), "+v"(at8[i].skip));
            if constexpr (H) keep(wn[i]);
        }
        if constexpr (kLean) fetch(row, gate_row);
        // per value: a = gy + r_y gu w_next, n_y, and for the block's side q
        const float ry = ryr, rh = rhr;
        float a[I][8];
        V y[I], h[B], g[B];
        uint32_t mask[B];
        float sum[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const uint32_t own8 = 0xFFu << at8[i].skip;
            if constexpr (kLean) wn[i] = ones8<T>(p.wn, at8[i]);
            y[i] = yr[i];
            if constexpr (H) {
                h[i] = hr[i];
                g[i] = gr[i];
                mask[i] = mask8<TAIL>(p.drop, row, at8[i].c);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float gu = at(gur[i], j), wnj = at(wn[i], j), ny = at(y[i], j) * ry, e = gu * ny;
                const bool own = !TAIL || (own8 >> j & 1);
                sum[0] += own ? wnj * e : 0.0f;
                sn[i][j] += e;
                a[i][j] = at(gyr[i], j) + ry * (gu * wnj);
                if constexpr (H) {
                    const float kg = at(sc[i], j) * at(w[i], j) * at(g[i], j);
                    const float q = own && (mask[i] >> j & 1) ? kg * (at(h[i], j) * rh) : 0.0f;
                    sum[1] += a[i][j] * q;
                    sum[2] += ny * q;
                }
            }
            if constexpr (I == 1 || H) {   // the next half starts from the loaded values
                keep(y[i]);
                if constexpr (H) {
                    keep(h[i]);
                    keep(g[i]);
                    keep(w[i]);
                    keep(sc[i]);
                }
            }
        }
        const bool last = k.last(rw);
        k.advance(p, rw);
        if (!kLean && k.row < p.N) fetch(k.row, k.gate_row);
        if constexpr (H) {
            worker_sum<TPR, 3>(sum, s, turn);
        } else {
            float one[1] = {sum[0]};
            worker_sum<TPR, 1>(one, s, turn);
            sum[0] = one[0];
        }
        const float fs = H ? p.drop.threshold ? p.drop.scale : 1.0f : 0.0f;
        const float c1 = sum[0] / (float)D, c2 = fs * (sum[1] - ry * c1 * sum[2]) / (float)D, ryc1 = ry * c1;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            if (at8[i].skip == 8) continue;
            float gx[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) gx[j] = a[i][j] - at(y[i], j) * ry * ryc1;
            if (p.gx) put8<T>((T*)p.gx + row * D, at8[i], gx);
            if constexpr (H) {
                float gh[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool in = mask[i] >> j & 1;
                    const float kg = at(sc[i], j) * at(w[i], j) * at(g[i], j), nh = at(h[i], j) * rh;
                    const float d = in ? gx[j] * fs : 0.0f;     // with respect to scale gate N(h)
                    gh[j] = rh * (d * kg - nh * c2);
                    sm[i][j] += in ? d * nh : 0.0f;
                }
                put8<T>((T*)p.gh + row * D, at8[i], gh);
                if (last) {
                    float gg[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        gg[j] = at(sc[i], j) * at(w[i], j) * sm[i][j];
                        sg[i][j] += at(g[i], j) * sm[i][j];
                        sm[i][j] = 0.0f;
                    }
                    if (p.ggate && rw.parts > 1) {
                        float* to = p.partial + worker * D + at8[i].c;   // gate rows' parts come first
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            to[j] = gg[j];
                    } else if (p.ggate) {
                        put8<T>((T*)p.ggate + gate_row * D, at8[i], gg);
                    }
                }
            }
        }
    }

    // column sums of the work-group
    const int64_t gates_at = H && rw.parts > 1 ? rw.workers * D : 0;
    float* out = p.partial + gates_at + (int64_t)blockIdx.x * kSums * D;
#pragma unroll
    for (int m = 0; m < kSums; ++m) {
        if constexpr (kWorkers > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (at8[i].skip < 8) cols[sub * (TPR * I * 8) + at8[i].c + j] = m == kSums - 1 ? sn[i][j] : sg[H ? i : 0][j];
            __syncthreads();
            for (int c = threadIdx.x; c < D; c += kGroup) {
                float v = 0.0f;
#pragma unroll
                for (int w = 0; w < kWorkers; ++w) v += cols[w * (TPR * I * 8) + c];
                out[(int64_t)m * D + c] = v;
            }
        } else {
#pragma unroll
            for (int i = 0; i < I; ++i) {
                if (at8[i].skip == 8) continue;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    out[(int64_t)m * D + at8[i].c + j] = m == kSums - 1 ? sn[i][j] : sg[H ? i : 0][j];
            }
        }
    }
}

// The work-groups' column sums added up, then, by the work-groups after those, the parts of each gate row: a work-group
// takes 1024 / strands columns by so many strands of rows.  Every sum is taken in a fixed order.  (1001 sets of 2 x 1089
// sums: 7.4 us, 7.8 with half the strands; beside them 32 gate rows of 4096 in 16 parts: 7.1 us with a strand for these, 11.2
// with sixteen, which a gate row of 1000 columns in a thousand parts needs.)
struct Join { int sums, strands, gate_strands; };   // strands: as powers of two
template <typename T>
__global__ __launch_bounds__(1024) void norm_join_kernel(NormArgs p, Rows rw, int64_t groups, Join jn) {
    const int64_t D = p.width, sum_blocks = (D + (1024 >> jn.strands) - 1) >> (10 - jn.strands);
    const bool gates = blockIdx.x >= sum_blocks * jn.sums;
    const int shift = 10 - (gates ? jn.gate_strands : jn.strands), columns = 1 << shift, strands = 1024 >> shift;
    const uint32_t blocks = (uint32_t)((D + columns - 1) >> shift), id = gates ? blockIdx.x - (uint32_t)sum_blocks * jn.sums : blockIdx.x;
    const int64_t job = id / blocks;
    const int strand = threadIdx.x >> shift;
    const int64_t c = ((int64_t)(id % blocks) << shift) + (threadIdx.x & (columns - 1));
    const float* from;
    int64_t n;
    const bool split = jn.sums == 2 && rw.parts > 1;
    if (gates) {
        from = p.partial + job * rw.parts * D + c;
        // the last gate row may have fewer rows: the workers beyond them wrote nothing
        const int64_t left = p.N - job * p.rows_per_gate;
        n = left < rw.parts ? left : rw.parts;
    } else {
        from = p.partial + (split ? rw.workers * D : 0) + job * D + c;
        n = groups;
    }
    const int64_t step = gates ? D : jn.sums * D;
    float v = 0.0f, u[8] = {};
    if (c < D) {
        int64_t i = strand;
        for (; i + 7 * strands < n; i += 8 * strands)   // eight loads in flight
#pragma unroll
            for (int k = 0; k < 8; ++k) u[k] += from[(i + strands * k) * step];
        for (; i < n; i += strands) v += from[i * step];
#pragma unroll
        for (int k = 0; k < 8; ++k) v += u[k];
    }
    __shared__ float s[1024];
    s[threadIdx.x] = v;
    __syncthreads();
    if (strand || c >= D) return;
#pragma unroll 8
    for (int k = 1; k < strands; ++k) v += s[(k << shift) + threadIdx.x];
    if (gates) {
        ((T*)p.ggate)[job * D + c] = (T)v;
    } else if (job == jn.sums - 1) {
        if (p.gwn) ((T*)p.gwn)[c] = (T)v;
    } else {
        if (p.gw) ((T*)p.gw)[c] = (T)(v * load<T>(p.scale, c, 1.0f));
        if (p.gscale) ((T*)p.gscale)[c] = (T)(v * load<T>(p.w, c, 1.0f));
    }
}

// Threads a row and turns for a width; none below a chunk and above what registers hold.  The backward pass of a block's
// side takes one turn, and two above 4096 columns of 16-bit arrays (247 registers; 4000 x 8000 in bf16: 135 us, 165 with 1024
// threads and no loads ahead, 308 by the two kernels for wide rows); 32-bit ones do not fit there (294 us with 1024 threads at
// 4000 x 6000, 300 by the two kernels).
enum Pass { kForward, kBackward, kBackwardBlock };
struct Shape { int tpr, turns; };
inline Shape shape_of(int64_t width, Pass pass, int bytes) {
    const int64_t chunks = (width + 7) / 8;
    if (width < 8) return {0, 0};   // row8 reads eight values
    for (int t : {8, 16, 32, 64})
        if (chunks <= t) return {t, 1};
    if (pass == kBackwardBlock) {
        for (int t : {128, 192, 256, 512})
            if (chunks <= t) return {t, 1};
        return chunks <= 1024 && bytes == 2 ? Shape{512, 2} : Shape{0, 0};
    }
    if (chunks <= 128) return {64, 2};
    if (chunks <= 192) return {192, 1};
    if (chunks <= 256) return {256, 1};
    for (int t : {256, 512, 1024})
        if (chunks <= 2 * t) return {t, 2};
    return {0, 0};
}

// Workers of the column kernel: about four work-groups a compute unit over all columns.
inline int64_t column_blocks(int64_t width) { return (width + 8 * kThreads - 1) / (8 * kThreads); }

inline Rows rows_of(const Shape& sh, int64_t width, int64_t N, int64_t rows_per_gate, int bytes, bool block) {
    const int64_t wide = 1024 / column_blocks(width);
    // as many workers as the compute units hold at once
    const int per = sh.tpr ? group_of(sh.tpr) / sh.tpr : 1;
    const int held = sh.tpr ? 256 * backward_waves(bytes, sh.tpr, sh.turns, block) / group_of(sh.tpr) * per : 0;
    const int64_t want = sh.tpr ? 256 * held : wide > 1 ? wide : 1;
    // and of many rows two or four each, or the joining kernel has more to read than the others save (8192 x 289: 2 us)
    const int64_t least = N >= 4096 ? 4 : N >= 256 ? 2 : 1;
    // (no more workers than are held: a second round of a few would take as long as the first)
    const int64_t gates = N > 0 ? (N + rows_per_gate - 1) / rows_per_gate : 0;
    Rows out = {1, 0};
    if (gates > 0 && gates < want) {
        const int64_t most = ((rows_per_gate < N ? rows_per_gate : N) + least - 1) / least;
        const int64_t fit = sh.tpr ? want / gates : (want + gates - 1) / gates;
        out.parts = fit < most ? fit : most;
    }
    int64_t each = (gates + want - 1) / want;
    if (each < (least + rows_per_gate - 1) / rows_per_gate) each = (least + rows_per_gate - 1) / rows_per_gate;
    out.workers = out.parts > 1 ? gates * out.parts : (gates + each - 1) / each;
    return out;
}

inline int64_t groups_for(const Rows& r, const Shape& sh) {
    const int64_t per = sh.tpr ? group_of(sh.tpr) / sh.tpr : 1;
    return (r.workers + per - 1) / per;
}

// A thread a block of eight columns (one call of the generator) and turn; the row and block of its next turn follow
// from the last one's without a division.  Bound by HBM: 5.2 TB/s at 8192 x 16384 in bf16 (103 us); 6 us at 8192 x 289 in fp32.
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
    const Shape sh = shape_of(a.width, kForward, (int)sizeof(T));
    if (sh.tpr == 0) {
        norm_forward_kernel<T><<<dim3(row_groups(a.N)), kThreads, 0, s>>>(a);
        return (int)hipGetLastError();
    }
    const bool tail = a.width % 8 != 0, block = a.h != nullptr;
    // as many work-groups as the compute units hold walk the rows
    const int64_t per = group_of(sh.tpr) / sh.tpr, all = (a.N + per - 1) / per;
    const int64_t most = 256 * (256 * forward_waves(sizeof(T), sh.tpr, sh.turns, block) / group_of(sh.tpr));
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
    const Shape sh = shape_of(a.width, block ? kBackwardBlock : kBackward, (int)sizeof(T));
    const Rows rw = rows_of(sh, a.width, a.N, block ? a.rows_per_gate : 1, (int)sizeof(T), block);
    const int64_t groups = groups_for(rw, sh);
    if (sh.tpr == 0 && groups > 0) {
        norm_means_kernel<T><<<dim3(row_groups(a.N)), kThreads, 0, s>>>(a, rw);
        norm_columns_kernel<T><<<dim3((unsigned)groups, (unsigned)column_blocks(a.width)), kThreads, 0, s>>>(a, rw);
    } else if (groups > 0 && block) {
#define FFN_BLOCK(TPR, I)                                                                                           \
    if (tail) norm_backward_rows<T, TPR, I, true, true><<<dim3((unsigned)groups), group_of(TPR), 0, s>>>(a, rw);    \
    else norm_backward_rows<T, TPR, I, false, true><<<dim3((unsigned)groups), group_of(TPR), 0, s>>>(a, rw)
        switch (sh.tpr * sh.turns) {
            case 8: FFN_BLOCK(8, 1); break;
            case 16: FFN_BLOCK(16, 1); break;
            case 32: FFN_BLOCK(32, 1); break;
            case 64: FFN_BLOCK(64, 1); break;
            case 128: FFN_BLOCK(128, 1); break;
            case 192: FFN_BLOCK(192, 1); break;
            case 256: FFN_BLOCK(256, 1); break;
            case 512: FFN_BLOCK(512, 1); break;
            default:
                if constexpr (sizeof(T) == 2) {
                    FFN_BLOCK(512, 2);
                }
                break;
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
        // one strand where a gate row has few parts
        const Join jn = {block ? 2 : 1, 5, rw.parts > 64 ? 4 : 0};
        auto blocks = [&](int strands) { return (a.width + (1024 >> strands) - 1) >> (10 - strands); };
        const int64_t gates = a.ggate && rw.parts > 1 ? (a.N + a.rows_per_gate - 1) / a.rows_per_gate : 0;
        norm_join_kernel<T><<<dim3((unsigned)(jn.sums * blocks(jn.strands) + gates * blocks(jn.gate_strands))), 1024, 0, s>>>(a, rw, groups, jn);
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

inline int64_t workspace_floats(int64_t width, int64_t N, int64_t rows_per_gate, bool residual, int bytes) {
    const Shape sh = shape_of(width, residual ? kBackwardBlock : kBackward, bytes);
    const Rows rw = rows_of(sh, width, N, residual ? rows_per_gate : 1, bytes, residual);
    return (residual && rw.parts > 1 ? rw.workers * width : 0) + groups_for(rw, sh) * (residual ? 2 : 1) * width + (sh.tpr ? 0 : 2 * N);
}

}  // namespace
}  // namespace ffn
