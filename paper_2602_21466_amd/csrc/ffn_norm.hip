// Norms before and after a block with its gate and residual scale, and dropout.
#include "ffn_device.h"

namespace ffn {
namespace {

using namespace dev;

constexpr int kThreads = 256;
constexpr int kChunk = 64;   // rows whose column sums one work-group of the backward pass holds

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

// Terms of one value of the backward pass, given the row's means.
struct Terms { float gx, ny, nh, f, g, s; };
template <typename T> __device__ __forceinline__ Terms terms(const NormArgs& p, int64_t row, int64_t c, float ry, float rh, float c1) {
    Terms t = {};
    t.gx = p.gy ? to_f32(((const T*)p.gy)[row * p.width + c]) : 0.0f;
    if (p.gu) {
        t.ny = to_f32(((const T*)p.y)[row * p.ldx + c]) * ry;
        t.gx += ry * (to_f32(((const T*)p.gu)[row * p.ldg + c]) * load<T>(p.wn, c, 1.0f) - t.ny * c1);
    }
    if (p.h) {
        t.f = factor(p.drop, row, c);
        t.g = load<T>(p.gate, row / p.rows_per_gate * p.width + c, 1.0f);
        t.s = load<T>(p.scale, c, 1.0f);
        t.nh = to_f32(((const T*)p.h)[row * p.width + c]) * rh;
    }
    return t;
}

// The two means of each row: of (gu w_next) n_y, and of (d/dN(h)) w n_h.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_means_kernel(NormArgs p) {
    __shared__ float s[kThreads / 64];
    const int64_t D = p.width;
    for (int64_t row = blockIdx.x; row < p.N; row += gridDim.x) {
    const float ry = p.gu ? p.rstd_y[row] : 0.0f, rh = p.h ? p.rstd_h[row] : 0.0f;
    float c1 = 0.0f, c2 = 0.0f;
    if (p.gu) {
        for (int64_t c = threadIdx.x; c < D; c += kThreads)
            c1 += to_f32(((const T*)p.gu)[row * p.ldg + c]) * load<T>(p.wn, c, 1.0f) * (to_f32(((const T*)p.y)[row * p.ldx + c]) * ry);
        c1 = group_sum(c1, s) / (float)D;
    }
    if (p.h) {
        for (int64_t c = threadIdx.x; c < D; c += kThreads) {
            const Terms t = terms<T>(p, row, c, ry, rh, c1);
            if (t.f != 0.0f) c2 += t.gx * t.s * t.g * t.f * load<T>(p.w, c, 1.0f) * t.nh;
        }
        c2 = group_sum(c2, s) / (float)D;
    }
    if (threadIdx.x == 0) {
        p.partial[row] = c1;
        p.partial[p.N + row] = c2;
    }
    }
}

// A thread a column: the rows' gradients, and the column sums of kChunk rows (of one gate row's where ggate is asked for).
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_grad_kernel(NormArgs p) {
    const int64_t D = p.width, c = (int64_t)blockIdx.y * kThreads + threadIdx.x;
    if (c >= D) return;
    const int64_t r0 = (int64_t)blockIdx.x * kChunk, r1 = r0 + kChunk < p.N ? r0 + kChunk : p.N;
    float w = load<T>(p.w, c, 1.0f), sw = 0.0f, ss = 0.0f, sn = 0.0f;
    for (int64_t row = r0; row < r1; ++row) {
        const float ry = p.gu ? p.rstd_y[row] : 0.0f, rh = p.h ? p.rstd_h[row] : 0.0f;
        const float c1 = p.partial[row], c2 = p.partial[p.N + row];
        const Terms t = terms<T>(p, row, c, ry, rh, c1);
        if (p.gx) ((T*)p.gx)[row * D + c] = (T)t.gx;
        if (p.gu) sn += to_f32(((const T*)p.gu)[row * p.ldg + c]) * t.ny;
        if (p.h) {
            const float gv = t.f == 0.0f ? 0.0f : t.gx * t.s * t.g * t.f;
            ((T*)p.gh)[row * D + c] = (T)(rh * (gv * w - t.nh * c2));
            sw += gv * t.nh;
            if (t.f != 0.0f) ss += t.gx * t.g * t.f * (t.nh * w);
        }
    }
    float* out = p.partial + 2 * p.N + (int64_t)blockIdx.x * 3 * D;
    out[c] = sw;
    out[D + c] = ss;
    out[2 * D + c] = sn;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void norm_sum_kernel(NormArgs p, int64_t chunks) {
    const int64_t D = p.width, c = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (c >= D) return;
    void* to[3] = {p.gw, p.gscale, p.gwn};
    for (int j = 0; j < 3; ++j) {
        if (!to[j]) continue;
        float v = 0.0f;
        for (int64_t i = 0; i < chunks; ++i) v += p.partial[2 * p.N + (i * 3 + j) * D + c];
        ((T*)to[j])[c] = (T)v;
    }
}

// The gate's gradient: a thread a column of one gate row, over the rows that share it.
template <typename T>
__global__ __launch_bounds__(kThreads) void gate_grad_kernel(NormArgs p) {
    const int64_t D = p.width, c = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (c >= D) return;
    const int64_t gates = (p.N + p.rows_per_gate - 1) / p.rows_per_gate;
    for (int64_t k = blockIdx.y; k < gates; k += gridDim.y) {
        const int64_t r0 = k * p.rows_per_gate, r1 = r0 + p.rows_per_gate < p.N ? r0 + p.rows_per_gate : p.N;
        float v = 0.0f;
        for (int64_t row = r0; row < r1; ++row) {
            const Terms t = terms<T>(p, row, c, p.gu ? p.rstd_y[row] : 0.0f, p.rstd_h[row], p.partial[row]);
            if (t.f != 0.0f) v += t.gx * t.s * t.f * (t.nh * load<T>(p.w, c, 1.0f));
        }
        ((T*)p.ggate)[k * D + c] = (T)v;
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const T* x, int64_t ldx, T* y, int64_t ldy, int64_t N, int64_t width,
                                                           DropArgs d) {
    const int64_t blocks = (width + 7) / 8, total = N * blocks;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
        const int64_t row = i / blocks, b = i - row * blocks;
        const Words q = philox((uint32_t)b, (uint32_t)row, d.offset, d.seed);
        for (int j = 0; j < 8 && b * 8 + j < width; ++j) {
            const float v = to_f32(x[row * ldx + b * 8 + j]);
            y[row * ldy + b * 8 + j] = (T)(kept(q, j, d.threshold) ? v * d.scale : 0.0f);
        }
    }
}

inline unsigned row_groups(int64_t N) { return (unsigned)(N < (1 << 20) ? N : 1 << 20); }

template <typename T> int forward(const NormArgs& a, hipStream_t s) {
    norm_forward_kernel<T><<<dim3(row_groups(a.N)), kThreads, 0, s>>>(a);
    return (int)hipGetLastError();
}

template <typename T> int backward(const NormArgs& a, hipStream_t s) {
    const int64_t chunks = (a.N + kChunk - 1) / kChunk;
    const unsigned cols = (unsigned)((a.width + kThreads - 1) / kThreads);
    if (a.N > 0) {
        norm_means_kernel<T><<<dim3(row_groups(a.N)), kThreads, 0, s>>>(a);
        if (a.ggate) {
            const int64_t gates = (a.N + a.rows_per_gate - 1) / a.rows_per_gate;
            gate_grad_kernel<T><<<dim3(cols, (unsigned)(gates < 65535 ? gates : 65535)), kThreads, 0, s>>>(a);
        }
        norm_grad_kernel<T><<<dim3((unsigned)chunks, cols), kThreads, 0, s>>>(a);
    }
    norm_sum_kernel<T><<<dim3(cols), kThreads, 0, s>>>(a, chunks);
    return (int)hipGetLastError();
}

}  // namespace

int64_t norm_workspace_floats(int64_t width, int64_t N, int64_t, bool) {
    return 2 * N + (N + kChunk - 1) / kChunk * 3 * width;
}

int launch_norm_forward(const NormArgs& a, int32_t dtype, void* stream) {
    hipStream_t s = (hipStream_t)stream;
    return dtype == FFN_FP32 ? forward<float>(a, s) : dtype == FFN_BF16 ? forward<bf16>(a, s) : forward<fp16>(a, s);
}

int launch_norm_backward(const NormArgs& a, int32_t dtype, void* stream) {
    hipStream_t s = (hipStream_t)stream;
    return dtype == FFN_FP32 ? backward<float>(a, s) : dtype == FFN_BF16 ? backward<bf16>(a, s) : backward<fp16>(a, s);
}

int launch_dropout(const void* x, int64_t ldx, void* y, int64_t ldy, int64_t N, int64_t width, int32_t dtype,
                   const DropArgs& d, void* stream) {
    hipStream_t s = (hipStream_t)stream;
    const int64_t groups = (N * ((width + 7) / 8) + kThreads - 1) / kThreads;
    const dim3 grid((unsigned)(groups < 65536 ? groups : 65536));
    if (dtype == FFN_FP32) dropout_kernel<float><<<grid, kThreads, 0, s>>>((const float*)x, ldx, (float*)y, ldy, N, width, d);
    else if (dtype == FFN_BF16) dropout_kernel<bf16><<<grid, kThreads, 0, s>>>((const bf16*)x, ldx, (bf16*)y, ldy, N, width, d);
    else dropout_kernel<fp16><<<grid, kThreads, 0, s>>>((const fp16*)x, ldx, (fp16*)y, ldy, N, width, d);
    return (int)hipGetLastError();
}

}  // namespace ffn
