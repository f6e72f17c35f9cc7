// The layer norm of fp16 arrays.
#include "ffn_layer.h"

namespace ffn {
int launch_layer_forward_fp16(const LayerArgs& a, void* stream) { return layer_forward<dev::fp16>(a, (hipStream_t)stream); }
int launch_layer_backward_fp16(const LayerArgs& a, void* stream) { return layer_backward<dev::fp16>(a, (hipStream_t)stream); }
}  // namespace ffn
