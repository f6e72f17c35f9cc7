// Launch descriptions shared by ffn_plan.cpp (the C ABI, checks, workspaces)
// and the kernels of the feed-forward sublayer.  Internal.
#pragma once

#include <cstdint>

#include "ffn.h"

namespace ffn {

// ---------------------------------------------------------------- matrix products
// C(m, n) = sum_k A(m, k) B(n, k); see ffn_tile.h.
enum Epilogue : int32_t {
    kStore = 0,      // C
    kGate = 1,       // B holds the gate's N rows, then the up projection's: H = act(G) * U; G, U kept in `saved`
    kGateGrad = 2,   // the sum is dH: dG, dU into C [M, 2 N], H into `h`
    kPartial = 3,    // 32-bit partial sums of one split of k
    kEither = 4,     // C, or the 32-bit sums of a part of an expert's rows
};

// Operands and results of one launch.  Strides in elements; operands start on 16 bytes, with strides that are
// multiples of 16 bytes, and, along k, zeros up to the next multiple.
struct TileArgs {
    const void *a, *b;
    int64_t lda, ldb;
    int64_t M, N, K;
    int32_t act;
    int32_t tiles_m, tiles_n, splits;
    void* c;                              // kStore: C; kPartial: floats [splits, M, ldc]; kGate: H; kGateGrad: [dG dU]
    int64_t ldc;
    float* saved;                         // [M, 2 N]
    void* h;                              // kGateGrad: H
    int64_t ldh;
};

int launch_tile_bf16(const TileArgs& p, int32_t epilogue, bool a_cols, bool b_cols, int32_t tile, void* stream);
int launch_tile_fp16(const TileArgs& p, int32_t epilogue, bool a_cols, bool b_cols, int32_t tile, void* stream);
int launch_tile_fp32(const TileArgs& p, int32_t epilogue, bool a_cols, bool b_cols, int32_t tile, void* stream);

// The forward products for few rows (M <= kFewRows): C = X W^T (kStore) or the gated form (kGate: W holds the gate's
// N rows, then the up projection's).  Strides in elements of the arrays' type; any alignment.  See ffn_few.h.
constexpr int64_t kFewRows = 64;
struct FewArgs {
    const void *x, *w;
    int64_t ldx, ldw, M, N, K;
    void* c;
    int64_t ldc;
    float* saved;                         // kGate: [M, 2 N] or NULL
    int32_t act;
};
int launch_few_bf16(const FewArgs& p, int32_t epilogue, int32_t nr, int32_t waves, void* stream);
int launch_few_fp16(const FewArgs& p, int32_t epilogue, int32_t nr, int32_t waves, void* stream);
int launch_few_fp32(const FewArgs& p, int32_t epilogue, int32_t nr, int32_t waves, void* stream);

// Partial sums of C = A W, W [K, N] of 32-bit values with row stride ldw, for M <= kFewRows and N >= 4: floats
// [splits, M, ldc].  See ffn_few_grad.hip.
struct FewGradArgs {
    const void *x, *w;
    int64_t ldx, ldw, M, N, K;
    float* c;
    int64_t ldc;
    int32_t splits, waves;
};
int launch_few_grad(const FewGradArgs& p, void* stream);

// out[i, j] = sum over splits of partial[s, i, j] (rows of ld floats), N columns, out contiguous.
int launch_join(const float* partial, int64_t ld, int32_t splits, int64_t M, int64_t N, void* out, int32_t dtype, void* stream);

int launch_zero(void* p, int64_t bytes, void* stream);

// The same for the gate's epilogues (p as for the tile launch: p.c is H or [dG dU], p.splits the parts).
int launch_join_gate(const TileArgs& p, int32_t epilogue, const float* partial, int64_t ld, int32_t dtype, void* stream);

// [rows, width] with row stride ld -> the same with row stride `to_ld`, a multiple of 8 (zeros from width on).  Up to
// four matrices a launch.
struct PackJob {
    const void* from;
    void* to;
    int64_t ld, rows, width, to_ld;
    int32_t end;                          // work-groups up to here; set by the launcher
};
struct PackJobs {
    PackJob job[4];
    int32_t n;
};
int launch_pack(PackJobs jobs, int32_t dtype, void* stream);

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

int64_t norm_workspace_floats(int64_t width, int64_t N, int64_t rows_per_gate, bool residual, int bytes);

#define FFN_NORM_LAUNCHERS(TYPE)                                                                                     \
    int launch_norm_forward_##TYPE(const NormArgs& a, void* stream);                                                 \
    int launch_norm_backward_##TYPE(const NormArgs& a, void* stream);                                                \
    int launch_dropout_##TYPE(const void* x, int64_t ldx, void* y, int64_t ldy, int64_t N, int64_t width,            \
                              const DropArgs& d, void* stream);
FFN_NORM_LAUNCHERS(fp32)
FFN_NORM_LAUNCHERS(bf16)
FFN_NORM_LAUNCHERS(fp16)
#undef FFN_NORM_LAUNCHERS

}  // namespace ffn
