// Launch descriptions shared by ffn_plan.cpp (the C ABI, checks, workspaces)
// and the kernels of the feed-forward sublayer.  Internal.
#pragma once

#include <cstdint>

#include "ffn.h"

namespace ffn {

// ---------------------------------------------------------------- matrix products
// C[m, n] = sum_k A(m, k) B(n, k).  A stored [M, K] (row stride lda) or, with
// a_cols, [K, M]; likewise B.
enum Epilogue : int32_t {
    kStore = 0,      // C
    kGate = 1,       // B holds the gate's N rows, then the up projection's: H = act(G) * U; G, U kept in `saved`
    kGateGrad = 2,   // acc is dH: dG, dU into C [M, 2 N], H into `h`
};

struct GemmArgs {
    const void *a, *b;
    int64_t lda, ldb;
    int32_t a_cols, b_cols;
    int64_t M, N, K;
    void* c;
    int64_t ldc;
    int32_t epilogue, act;
    void* saved;     // kGate: output or NULL; kGateGrad: input; [M, 2 N] floats
    void* h;         // kGateGrad: [M, N]
};

int launch_gemm(const GemmArgs& a, int32_t dtype, void* stream);

// ---------------------------------------------------------------- norms and dropout

struct DropArgs {
    uint32_t threshold;   // of 65536; 0: keep everything
    float scale;          // 65536 / (65536 - threshold), 0 where everything is dropped
    uint64_t seed, offset;
};

struct NormArgs {
    int64_t width, N, rows_per_gate;
    float eps;
    DropArgs drop;
    // forward: x, h (NULL: no block output, u = N(x; wn)), w, gate, scale, wn -> y, u, rstd_h, rstd_y
    const void *x, *h, *w, *gate, *scale, *wn;
    int64_t ldx, ldu;
    void *y, *u;
    float *rstd_h, *rstd_y;
    // backward: y (ldx), gy, gu (ldg) -> gx, gh, column sums
    const void *gy, *gu;
    int64_t ldg;
    void *gx, *gh, *gw, *ggate, *gscale, *gwn;
    float* partial;       // workspace
};

int launch_norm_forward(const NormArgs& a, int32_t dtype, void* stream);
int launch_norm_backward(const NormArgs& a, int32_t dtype, void* stream);
int64_t norm_workspace_floats(int64_t width, int64_t N, int64_t rows_per_gate, bool residual);

int launch_dropout(const void* x, int64_t ldx, void* y, int64_t ldy, int64_t N, int64_t width, int32_t dtype,
                   const DropArgs& d, void* stream);

}  // namespace ffn
