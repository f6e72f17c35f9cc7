// The layer norm of bf16 arrays.
#include "ffn_layer.h"

namespace ffn {
int launch_layer_forward_bf16(const LayerArgs& a, void* stream) { return layer_forward<dev::bf16>(a, (hipStream_t)stream); }
int launch_layer_backward_bf16(const LayerArgs& a, void* stream) { return layer_backward<dev::bf16>(a, (hipStream_t)stream); }
}  // namespace ffn
