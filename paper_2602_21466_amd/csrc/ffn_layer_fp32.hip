// The layer norm of fp32 arrays.
#include "ffn_layer.h"

namespace ffn {
int launch_layer_forward_fp32(const LayerArgs& a, void* stream) { return layer_forward<float>(a, (hipStream_t)stream); }
int launch_layer_backward_fp32(const LayerArgs& a, void* stream) { return layer_backward<float>(a, (hipStream_t)stream); }
int64_t layer_workspace_floats(int64_t width, int64_t N, int bytes) { return layer_floats(width, N, bytes); }   // (of any type)
}  // namespace ffn
