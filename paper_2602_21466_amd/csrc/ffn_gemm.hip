// Packing of operands for the tiled products, and the joining of their split sums.
#include "ffn_tile.h"

namespace ffn {
namespace {

using namespace dev;

constexpr int kThreads = 256;

// A thread a chunk of eight values of the packed rows.
template <typename T>
__global__ __launch_bounds__(kThreads) void pack_kernel(const T* from, int64_t ld, int64_t rows, int64_t width, uint16_t* to,
                                                        int64_t to_ld, int64_t plane) {
    const int64_t chunks = to_ld >> 3, total = rows * chunks;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
        const int64_t row = i / chunks, c = (i - row * chunks) * 8;
        const T* f = from + row * ld + c;
        T v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < width ? f[j] : (T)0.0f;
        uint16_t* t = to + row * to_ld + c;
        if constexpr (sizeof(T) == 4) {
            s16x8 o[3];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint16_t q[3];
                planes_of(v[j], q);
                o[0][j] = (short)q[0];
                o[1][j] = (short)q[1];
                o[2][j] = (short)q[2];
            }
#pragma unroll
            for (int k = 0; k < 3; ++k) *(s16x8*)(t + k * plane) = o[k];
        } else {
            s16x8 o;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = __builtin_bit_cast(short, v[j]);
            *(s16x8*)t = o;
        }
    }
}

// Splits are added in order: the result does not depend on when they were done.
template <typename Out>
__global__ __launch_bounds__(kThreads) void join_kernel(const float* partial, int64_t ld, int splits, int64_t M, int64_t N, Out* out) {
    const int64_t quads = (N + 3) >> 2, total = M * quads;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
        const int64_t row = i / quads, c = (i - row * quads) * 4;
        f32x4 v = {};
        for (int s = 0; s < splits; ++s) v += *(const f32x4*)(partial + ((int64_t)s * M + row) * ld + c);
        store4<Out>(out + row * N, c, N, 0, v, (N & 3) == 0);
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

int launch_pack(const void* from, int64_t ld, int64_t rows, int64_t width, int32_t dtype, void* to, int64_t to_ld, int64_t plane,
                void* stream) {
    hipStream_t s = (hipStream_t)stream;
    const unsigned g = groups(rows * (to_ld >> 3));
    if (dtype == FFN_FP32) pack_kernel<float><<<g, kThreads, 0, s>>>((const float*)from, ld, rows, width, (uint16_t*)to, to_ld, plane);
    else pack_kernel<bf16><<<g, kThreads, 0, s>>>((const bf16*)from, ld, rows, width, (uint16_t*)to, to_ld, plane);   // bits alone
    return (int)hipGetLastError();
}

int launch_zero(void* p, int64_t bytes, void* stream) {
    zero_kernel<<<groups(bytes / 2), kThreads, 0, (hipStream_t)stream>>>((uint16_t*)p, bytes / 2);
    return (int)hipGetLastError();
}

int launch_join(const float* partial, int64_t ld, int32_t splits, int64_t M, int64_t N, void* out, int32_t dtype, void* stream) {
    hipStream_t s = (hipStream_t)stream;
    const unsigned g = groups(M * ((N + 3) >> 2));
    if (dtype == FFN_FP32) join_kernel<float><<<g, kThreads, 0, s>>>(partial, ld, splits, M, N, (float*)out);
    else if (dtype == FFN_BF16) join_kernel<bf16><<<g, kThreads, 0, s>>>(partial, ld, splits, M, N, (bf16*)out);
    else join_kernel<fp16><<<g, kThreads, 0, s>>>(partial, ld, splits, M, N, (fp16*)out);
    return (int)hipGetLastError();
}

}  // namespace ffn
