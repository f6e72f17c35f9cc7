// Norms and dropout of bf16 arrays.
#include "ffn_norm.h"

namespace ffn {
int launch_norm_forward_bf16(const NormArgs& a, void* stream) { return forward<dev::bf16>(a, (hipStream_t)stream); }
int launch_norm_backward_bf16(const NormArgs& a, void* stream) { return backward<dev::bf16>(a, (hipStream_t)stream); }
int launch_dropout_bf16(const void* x, int64_t ldx, void* y, int64_t ldy, int64_t N, int64_t width, const DropArgs& d, void* stream) {
    return drop<dev::bf16>(x, ldx, y, ldy, N, width, d, (hipStream_t)stream);
}
}  // namespace ffn
