// The experts' tiled products of fp16 arrays.
#include "ffn_experts.h"

namespace ffn {
int launch_expert_rows_fp16(const TileArgs& t, const Groups& g, int32_t epilogue, bool b_cols, int32_t tile, void* stream) {
    return dev::expert_rows<dev::fp16>(t, g, epilogue, b_cols, tile, (hipStream_t)stream);
}
int launch_expert_grads_fp16(const ExpertGrads& a, int32_t tile, void* stream) { return dev::expert_grads<dev::fp16>(a, tile, (hipStream_t)stream); }
}  // namespace ffn
