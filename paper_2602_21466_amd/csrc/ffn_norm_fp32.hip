// Norms and dropout of fp32 arrays.
#include "ffn_norm.h"

namespace ffn {
int launch_norm_forward_fp32(const NormArgs& a, void* stream) { return forward<float>(a, (hipStream_t)stream); }
int launch_norm_backward_fp32(const NormArgs& a, void* stream) { return backward<float>(a, (hipStream_t)stream); }
int launch_dropout_fp32(const void* x, int64_t ldx, void* y, int64_t ldy, int64_t N, int64_t width, const DropArgs& d, void* stream) {
    return drop<float>(x, ldx, y, ldy, N, width, d, (hipStream_t)stream);
}
int64_t norm_workspace_floats(int64_t width, int64_t N, int64_t rows_per_gate, bool residual, int bytes) {
    return workspace_floats(width, N, rows_per_gate, residual, bytes);   // (of any type)
}
}  // namespace ffn
