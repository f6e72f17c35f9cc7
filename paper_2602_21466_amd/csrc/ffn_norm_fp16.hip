// Norms and dropout of fp16 arrays.
#include "ffn_norm.h"

namespace ffn {
int launch_norm_forward_fp16(const NormArgs& a, void* stream) { return forward<dev::fp16>(a, (hipStream_t)stream); }
int launch_norm_backward_fp16(const NormArgs& a, void* stream) { return backward<dev::fp16>(a, (hipStream_t)stream); }
int launch_dropout_fp16(const void* x, int64_t ldx, void* y, int64_t ldy, int64_t N, int64_t width, const DropArgs& d, void* stream) {
    return drop<dev::fp16>(x, ldx, y, ldy, N, width, d, (hipStream_t)stream);
}
}  // namespace ffn
