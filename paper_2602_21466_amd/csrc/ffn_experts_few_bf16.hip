// The experts' forward products for few rows, bf16 arrays.
#include "ffn_experts_few.h"

namespace ffn {
int launch_expert_few_bf16(const FewArgs& p, const Groups& g, int32_t epilogue, int32_t rows, int32_t nr, int32_t waves, int64_t most, void* stream) {
    return dev::expert_few<dev::bf16>(p, g, epilogue, rows, nr, waves, most, (hipStream_t)stream);
}
}  // namespace ffn
