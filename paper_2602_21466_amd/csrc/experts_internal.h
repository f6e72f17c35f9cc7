// Launch descriptions shared by the C entries of the layer norm, the sorting of rows by expert and the experts' blocks
// (ffn_layer.cpp, experts_plan.cpp) and their kernels.  Internal.
#pragma once

#include <cstdint>

#include "experts.h"
#include "ffn_internal.h"

namespace ffn {

// ---------------------------------------------------------------- layer norm

struct LayerArgs {
    int64_t width, N;
    float eps;
    const void *x, *w, *b;
    int64_t ldx;
    void* u;                              // forward
    int64_t ldu;
    float* stats;                         // [2, N]: written forward, read backward
    const void* gu;                       // backward
    int64_t ldg;
    void *gx, *gw, *gb;
    float* partial;                       // workspace
};
int64_t layer_workspace_floats(int64_t width, int64_t N, int bytes);

#define FFN_LAYER_LAUNCHERS(TYPE)                                    \
    int launch_layer_forward_##TYPE(const LayerArgs& a, void* stream); \
    int launch_layer_backward_##TYPE(const LayerArgs& a, void* stream);
FFN_LAYER_LAUNCHERS(fp32)
FFN_LAYER_LAUNCHERS(bf16)
FFN_LAYER_LAUNCHERS(fp16)
#undef FFN_LAYER_LAUNCHERS

// ---------------------------------------------------------------- rows sorted by expert

struct SortArgs {
    const void* index;
    int32_t index_bytes, experts;
    int64_t slots, chunk;                 // slots a work-group
    int32_t groups;
    int32_t *place, *source, *offsets;
    int32_t* counts;                      // workspace [groups, experts]
};
int launch_sort(const SortArgs& a, void* stream);

struct RouteArgs {
    int64_t N, width, per_row, slots;
    const int32_t *place, *offsets;       // offsets: NULL where no rows behind the last are written
    int32_t experts;
    const float* weights;                 // NULL: ones
    const void *rows, *sorted;            // inputs [N, width] (stride ld) and [slots, width]
    int64_t ld;
    void *out_rows, *out_sorted;          // outputs; out_rows has stride ld_out, out_sorted ld_sorted (zeros behind width)
    int64_t ld_out, ld_sorted;
    float* grad_weights;
};
int launch_gather(const RouteArgs& a, int32_t dtype, void* stream);            // rows -> out_sorted
int launch_combine(const RouteArgs& a, int32_t dtype, void* stream);           // sorted -> out_rows
int launch_combine_backward(const RouteArgs& a, int32_t dtype, void* stream);  // rows (, sorted) -> out_sorted, grad_weights

// out_rows[n] = sum over k and over `splits` parts of the sorted rows place[n, k], floats [splits, slots, ld] in `sorted`.
int launch_combine_parts(const RouteArgs& a, int32_t splits, int32_t dtype, void* stream);

// ---------------------------------------------------------------- the experts' products

// Bytes that may be read behind the last expert's B where that is a copy.
constexpr int64_t kCopyRoom = 2;

// The runs of sorted rows that a launch's products are about.
struct Groups {
    const int32_t* offsets;
    int32_t experts;
    int64_t rows;                         // sorted rows there may be
    int64_t b_step;                       // bytes from one expert's B to the next's
    const void *a_end, *b_end;            // behind the last bytes that may be read of either operand
    int64_t b_shift;                      // bytes from where the last expert's B would be to where a copy of it is; 0: it is there
    int32_t chunk;                        // sums: rows of a part; 0: an expert's rows are one part
    const int32_t* source;                // rows of A are those of slots source[..] / per_row; NULL: they are in their order
    int32_t per_row;
    bool deep;                            // rows: no more tiles than compute units, by the mean (16-bit arrays, 128-wide tiles)
};
// Operands lie in memory as they are: rows start on any element, with anything behind them.
// C = A B^T for the rows of every expert with its own B: t.M is groups.rows, t.tiles_m as many tiles of rows as there can
// be (rows / tile + experts with a row).
int launch_expert_rows_bf16(const TileArgs& t, const Groups& g, int32_t epilogue, bool b_cols, int32_t tile, void* stream);
int launch_expert_rows_fp16(const TileArgs& t, const Groups& g, int32_t epilogue, bool b_cols, int32_t tile, void* stream);
int launch_expert_rows_fp32(const TileArgs& t, const Groups& g, int32_t epilogue, bool b_cols, int32_t tile, void* stream);
// The forward products for few rows an expert, as launch_few_* for a single block: x's rows by g.source, results in the
// sorted order; tiles of `rows` rows (16, 32 or 64), `most` of them at the most.
int launch_expert_few_bf16(const FewArgs& p, const Groups& g, int32_t epilogue, int32_t rows, int32_t nr, int32_t waves, int64_t most, void* stream);
int launch_expert_few_fp16(const FewArgs& p, const Groups& g, int32_t epilogue, int32_t rows, int32_t nr, int32_t waves, int64_t most, void* stream);
int launch_expert_few_fp32(const FewArgs& p, const Groups& g, int32_t epilogue, int32_t rows, int32_t nr, int32_t waves, int64_t most, void* stream);
// The gradients' products, in one launch; those whose t.a is NULL are left out.
//   0: C = A B^T for the rows of every expert as above (kPartial, B by columns)
//   1, 2: C_e = A_e^T B_e, the sum over the rows of expert e, for every expert: C [experts, t.M, t.N].  An expert of more than
//      g.chunk rows has as many parts; theirs go to partial[k - 1], floats [parts, t.M, t.N up to a multiple of four], for
//      launch_join_sums.  t.splits: parts there may be.
struct ExpertGrads {
    TileArgs t[3];
    Groups g[3];
    float* partial[2];
    int32_t order[3];                     // which product comes first, second, third
    int32_t end[3];                       // work-groups up to here, in that order; set by the launcher
};
int launch_expert_grads_bf16(const ExpertGrads& a, int32_t tile, void* stream);
int launch_expert_grads_fp16(const ExpertGrads& a, int32_t tile, void* stream);
int launch_expert_grads_fp32(const ExpertGrads& a, int32_t tile, void* stream);
int launch_join_sums(const ExpertGrads& a, int32_t dtype, void* stream);

// launch_join and launch_join_gate for as many of the rows as *limit says (NULL: all).
int launch_join_rows(const float* partial, int64_t ld, int32_t splits, int64_t M, int64_t N, void* out, int32_t dtype,
                     const int32_t* limit, void* stream);
int launch_join_gate_rows(const TileArgs& p, int32_t epilogue, const float* partial, int64_t ld, int32_t dtype,
                          const int32_t* limit, void* stream);

}  // namespace ffn
