// Packing of operands for the tiled products, and the joining of their split sums.
#include "experts_device.h"
#include "ffn_tile.h"

namespace ffn {
namespace {

using namespace dev;

constexpr int kThreads = 256;

// A thread a chunk of eight values of the packed rows; the work-groups are dealt to the matrices in turn.  Bound by HBM:
// 5.0 TB/s for 8192 x 3281 values of 32 bits (43 us).
template <typename T>
__global__ __launch_bounds__(kThreads) void pack_kernel(PackJobs jobs) {
    int k = 0, first = 0;
    while (k + 1 < jobs.n && (int)blockIdx.x >= jobs.job[k].end) first = jobs.job[k++].end;
    const PackJob& j = jobs.job[k];
    const int64_t stride = (int64_t)(j.end - first) * kThreads;
    const int64_t chunks = j.to_ld >> 3, total = j.rows * chunks;
    int64_t i = (int64_t)((int)blockIdx.x - first) * kThreads + threadIdx.x;
    int64_t row = i / chunks, at = i - row * chunks;
    const int64_t dr = stride / chunks, da = stride - dr * chunks;
    for (; i < total; i += stride) {
        const int64_t c = at * 8;
        const T* f = (const T*)j.from + row * j.ld + c;
        typedef T V __attribute__((ext_vector_type(8)));
        V v;
        if (c + 8 <= j.width) {
            __builtin_memcpy(&v, f, sizeof(v));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = c + e < j.width ? f[e] : (T)0.0f;
        }
        *(V*)((T*)j.to + row * j.to_ld + c) = v;
        row += dr;
        at += da;
        if (at >= chunks) { at -= chunks; ++row; }
    }
}

// Of M rows those that are finished: all, or as many as the device knows of (sorted by expert).
__device__ __forceinline__ int64_t rows_of(int64_t M, const int32_t* limit) {
    if (!limit) return M;
    const int64_t n = *limit;
    return n < 0 ? 0 : n < M ? n : M;
}

// Splits are added in order: the result does not depend on when they were done.  (3281 x 512 in 9 parts, fp32: 11 us.)
template <typename Out>
__global__ __launch_bounds__(kThreads) void join_kernel(const float* partial, int64_t ld, int splits, int64_t M, int64_t N, Out* out, const int32_t* limit) {
    const int64_t quads = (N + 3) >> 2, total = rows_of(M, limit) * quads;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
        const int64_t row = i / quads, c = (i - row * quads) * 4;
        f32x4 v = {};
#pragma unroll 8
        for (int s = 0; s < splits; ++s) v += *(const f32x4*)(partial + ((int64_t)s * M + row) * ld + c);
        store4<Out>(out + row * N, c, N, 0, v);
    }
}

// The joining of split sums with the gate's epilogues; the same arithmetic as the tiles' own.  kGate: the sums hold
// [G U] (2 N columns); kGateGrad: dH.  (8192 x 512, fp32: 23 us, 5.0 TB/s.)
template <typename T, int EPI>
__global__ __launch_bounds__(kThreads) void join_gate_kernel(TileArgs p, const float* partial, int64_t ld, const int32_t* limit) {
    const int64_t quads = (p.N + 3) >> 2, total = rows_of(p.M, limit) * quads;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
        const int64_t m = i / quads, n = (i - m * quads) * 4;
        f32x4 v = {}, u = {};
#pragma unroll 4
        for (int s = 0; s < p.splits; ++s) {
            const float* from = partial + ((int64_t)s * p.M + m) * ld;
            v += *(const f32x4*)(from + n);
            if constexpr (EPI == kGate) u += load4(from + p.N, n, p.N);
        }
        f32x4 h;
        if constexpr (EPI == kGate) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float a, da;
                activate<T>(p.act, v[e], a, da);
                h[e] = a * u[e];
            }
            store4<T>((T*)p.c + m * p.ldc, n, p.N, p.ldc, h);
            if (p.saved) {
                store4<float>(p.saved + m * 2 * p.N, n, p.N, 0, v);
                store4<float>(p.saved + m * 2 * p.N + p.N, n, p.N, 0, u);
            }
        } else {
            const f32x4 g = load4(p.saved + m * 2 * p.N, n, p.N);
            u = load4(p.saved + m * 2 * p.N + p.N, n, p.N);
            f32x4 dg, du;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float a, da;
                activate<T>(p.act, g[e], a, da);
                dg[e] = v[e] * u[e] * da;
                du[e] = v[e] * a;
                h[e] = a * u[e];
            }
            store_gate_grad<T>(p, m, n, dg, du, h);
        }
    }
}

// The parts of the experts that have more than one, added in order.  (3281 x 512 and 1024 x 128 of 5 experts in parts of 1024
// rows of 8192, fp32: 23 us.)
template <typename Out>
__global__ __launch_bounds__(kThreads) void join_sums_kernel(ExpertGrads a) {
    const TileArgs& p = a.t[1 + blockIdx.z];
    const Groups& g = a.g[1 + blockIdx.z];
    const float* partial = a.partial[blockIdx.z];
    if (!p.a) return;
    const int e = blockIdx.y, lane = threadIdx.x & 63;
    int first = 0, parts = 0;
    for (int e0 = 0; e0 <= e; e0 += 64) {
        Scan s;
        s.read(g, e0, lane, g.chunk, 1);
        const int rows = s.end - s.begin;
        if (e - e0 >= 64) {
            first += s.total();
            continue;
        }
        parts = Scan::tiles_of(__builtin_amdgcn_readlane(rows, e - e0), g.chunk, 1);
        first += __builtin_amdgcn_readlane(s.upto, e - e0) - parts;
    }
    if (parts == 1) return;
    if (parts > p.splits - first) parts = p.splits - first;   // (of offsets that ffn_route wrote there are no more)
    const int64_t ld = (p.N + 3) & ~3LL, quads = ld >> 2, total = p.M * quads, part = p.M * ld;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
        const int64_t row = i / quads, c = (i - row * quads) * 4;
        f32x4 v = {};
#pragma unroll 8
        for (int s = 0; s < parts; ++s) v += *(const f32x4*)(partial + (first + s) * part + row * ld + c);
        store4<Out>((Out*)p.c + (e * p.M + row) * p.N, c, p.N, 0, v);
    }
}

// (a kernel, not a memset: it may be captured in a graph)
__global__ __launch_bounds__(kThreads) void zero_kernel(uint16_t* p, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) p[i] = 0;
}

unsigned groups(int64_t n) {
    const int64_t g = (n + kThreads - 1) / kThreads;
    return (unsigned)(g < (1 << 20) ? g : 1 << 20);
}

}  // namespace

int launch_pack(PackJobs jobs, int32_t dtype, void* stream) {
    if (jobs.n == 0) return 0;
    int end = 0;
    for (int k = 0; k < jobs.n; ++k) {
        const int64_t n = (jobs.job[k].rows * (jobs.job[k].to_ld >> 3) + kThreads - 1) / kThreads;
        jobs.job[k].end = end += (int)(n < 4096 ? n : 4096);
    }
    hipStream_t s = (hipStream_t)stream;
    if (dtype == FFN_FP32) pack_kernel<float><<<end, kThreads, 0, s>>>(jobs);
    else pack_kernel<bf16><<<end, kThreads, 0, s>>>(jobs);   // bits alone
    return (int)hipGetLastError();
}

int launch_join_gate(const TileArgs& p, int32_t epilogue, const float* partial, int64_t ld, int32_t dtype, void* stream) {
    return launch_join_gate_rows(p, epilogue, partial, ld, dtype, nullptr, stream);
}

int launch_join_gate_rows(const TileArgs& p, int32_t epilogue, const float* partial, int64_t ld, int32_t dtype, const int32_t* limit, void* stream) {
    hipStream_t s = (hipStream_t)stream;
    const unsigned g = groups(p.M * ((p.N + 3) >> 2));
#define FFN_JOIN(T)                                                                                       \
    if (epilogue == kGate) join_gate_kernel<T, kGate><<<g, kThreads, 0, s>>>(p, partial, ld, limit);      \
    else join_gate_kernel<T, kGateGrad><<<g, kThreads, 0, s>>>(p, partial, ld, limit)
    if (dtype == FFN_FP32) { FFN_JOIN(float); }
    else if (dtype == FFN_BF16) { FFN_JOIN(bf16); }
    else { FFN_JOIN(fp16); }
#undef FFN_JOIN
    return (int)hipGetLastError();
}

int launch_join_sums(const ExpertGrads& a, int32_t dtype, void* stream) {
    hipStream_t s = (hipStream_t)stream;
    int64_t most = 0;
    for (int k : {1, 2})
        if (a.t[k].a && a.t[k].M * ((a.t[k].N + 3) >> 2) > most) most = a.t[k].M * ((a.t[k].N + 3) >> 2);
    const unsigned all = groups(most);
    const dim3 grid(all < 1024 ? all : 1024, (unsigned)(a.t[1].a ? a.g[1] : a.g[2]).experts, 2);
    if (dtype == FFN_FP32) join_sums_kernel<float><<<grid, kThreads, 0, s>>>(a);
    else if (dtype == FFN_BF16) join_sums_kernel<bf16><<<grid, kThreads, 0, s>>>(a);
    else join_sums_kernel<fp16><<<grid, kThreads, 0, s>>>(a);
    return (int)hipGetLastError();
}

int launch_zero(void* p, int64_t bytes, void* stream) {
    zero_kernel<<<groups(bytes / 2), kThreads, 0, (hipStream_t)stream>>>((uint16_t*)p, bytes / 2);
    return (int)hipGetLastError();
}

int launch_join(const float* partial, int64_t ld, int32_t splits, int64_t M, int64_t N, void* out, int32_t dtype, void* stream) {
    return launch_join_rows(partial, ld, splits, M, N, out, dtype, nullptr, stream);
}

int launch_join_rows(const float* partial, int64_t ld, int32_t splits, int64_t M, int64_t N, void* out, int32_t dtype, const int32_t* limit, void* stream) {
    hipStream_t s = (hipStream_t)stream;
    const unsigned g = groups(M * ((N + 3) >> 2));
    if (dtype == FFN_FP32) join_kernel<float><<<g, kThreads, 0, s>>>(partial, ld, splits, M, N, (float*)out, limit);
    else if (dtype == FFN_BF16) join_kernel<bf16><<<g, kThreads, 0, s>>>(partial, ld, splits, M, N, (bf16*)out, limit);
    else join_kernel<fp16><<<g, kThreads, 0, s>>>(partial, ld, splits, M, N, (fp16*)out, limit);
    return (int)hipGetLastError();
}

}  // namespace ffn
