// The experts' tiled products of fp32 arrays.
#include "ffn_experts.h"

namespace ffn {
int launch_expert_rows_fp32(const TileArgs& t, const Groups& g, int32_t epilogue, bool b_cols, int32_t tile, void* stream) {
    return dev::expert_rows<float>(t, g, epilogue, b_cols, tile, (hipStream_t)stream);
}
int launch_expert_grads_fp32(const ExpertGrads& a, int32_t tile, void* stream) { return dev::expert_grads<float>(a, tile, (hipStream_t)stream); }
}  // namespace ffn
