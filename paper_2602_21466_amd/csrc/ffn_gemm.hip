// Matrix products of the gated feed-forward block.
#include "ffn_device.h"

namespace ffn {
namespace {

using namespace dev;

constexpr int kTile = 64, kDepth = 16;

// One 64 x 64 tile of C a work-group of 256 threads, 4 x 4 values a thread; operands pass
// through LDS as 32-bit values, so every type, stride and alignment takes the same path.
template <typename T>
__global__ __launch_bounds__(256) void gemm_kernel(GemmArgs p) {
    __shared__ float sa[kDepth][kTile + 1], sb[2][kDepth][kTile + 1];
    const int64_t m0 = (int64_t)blockIdx.y * kTile, n0 = (int64_t)blockIdx.x * kTile;
    const int nb = p.epilogue == kGate ? 2 : 1;
    const int tm = threadIdx.x >> 4, tn = threadIdx.x & 15;
    const T *A = (const T*)p.a, *B = (const T*)p.b;
    float acc[2][4][4] = {};
    for (int64_t k0 = 0; k0 < p.K; k0 += kDepth) {
        for (int i = threadIdx.x; i < kTile * kDepth; i += 256) {
            const int r = p.a_cols ? i % kTile : i / kDepth, k = p.a_cols ? i / kTile : i % kDepth;
            const int64_t m = m0 + r, kk = k0 + k;
            sa[k][r] = m < p.M && kk < p.K ? to_f32(p.a_cols ? A[kk * p.lda + m] : A[m * p.lda + kk]) : 0.0f;
        }
        for (int j = 0; j < nb; ++j)
            for (int i = threadIdx.x; i < kTile * kDepth; i += 256) {
                const int r = p.b_cols ? i % kTile : i / kDepth, k = p.b_cols ? i / kTile : i % kDepth;
                const int64_t n = n0 + r, kk = k0 + k, row = n + j * p.N;
                sb[j][k][r] = n < p.N && kk < p.K ? to_f32(p.b_cols ? B[kk * p.ldb + row] : B[row * p.ldb + kk]) : 0.0f;
            }
        __syncthreads();
        for (int k = 0; k < kDepth; ++k)
            for (int j = 0; j < nb; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int y = 0; y < 4; ++y) acc[j][x][y] += sa[k][tm * 4 + x] * sb[j][k][tn * 4 + y];
        __syncthreads();
    }
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const int64_t m = m0 + tm * 4 + x, n = n0 + tn * 4 + y;
            if (m >= p.M || n >= p.N) continue;
            T* C = (T*)p.c;
            float* S = (float*)p.saved;
            float v, dv;
            if (p.epilogue == kStore) {
                C[m * p.ldc + n] = (T)acc[0][x][y];
            } else if (p.epilogue == kGate) {
                const float g = acc[0][x][y], u = acc[1][x][y];
                activate(p.act, g, v, dv);
                C[m * p.ldc + n] = (T)(v * u);
                if (S) {
                    S[m * 2 * p.N + n] = g;
                    S[m * 2 * p.N + p.N + n] = u;
                }
            } else {
                const float dh = acc[0][x][y], g = S[m * 2 * p.N + n], u = S[m * 2 * p.N + p.N + n];
                activate(p.act, g, v, dv);
                C[m * p.ldc + n] = (T)(dh * u * dv);
                C[m * p.ldc + p.N + n] = (T)(dh * v);
                ((T*)p.h)[m * p.N + n] = (T)(v * u);
            }
        }
}

}  // namespace

int launch_gemm(const GemmArgs& a, int32_t dtype, void* stream) {
    // the tiles' second index is held under the grid's limit by slabs of rows
    const int64_t slab = 65535LL * kTile;
    for (int64_t m = 0; m < a.M; m += slab) {
        GemmArgs p = a;
        const int64_t e = dtype == FFN_FP32 ? 4 : 2;
        p.M = a.M - m < slab ? a.M - m : slab;
        p.a = (const char*)a.a + (a.a_cols ? m : m * a.lda) * e;
        p.c = (char*)a.c + m * a.ldc * e;
        if (a.saved) p.saved = (char*)a.saved + m * 2 * a.N * 4;
        if (a.h) p.h = (char*)a.h + m * a.N * e;
        const dim3 grid((unsigned)((a.N + kTile - 1) / kTile), (unsigned)((p.M + kTile - 1) / kTile));
        hipStream_t s = (hipStream_t)stream;
        if (dtype == FFN_FP32) gemm_kernel<float><<<grid, 256, 0, s>>>(p);
        else if (dtype == FFN_BF16) gemm_kernel<bf16><<<grid, 256, 0, s>>>(p);
        else gemm_kernel<fp16><<<grid, 256, 0, s>>>(p);
        const hipError_t e2 = hipGetLastError();
        if (e2 != hipSuccess) return (int)e2;
    }
    return 0;
}

}  // namespace ffn
