// Forward products for few rows, bf16 arrays.
#include "ffn_few.h"

namespace ffn {
int launch_few_bf16(const FewArgs& p, int32_t epilogue, int32_t nr, int32_t waves, void* stream) {
    return dev::few<dev::bf16>(p, epilogue, nr, waves, (hipStream_t)stream);
}
}  // namespace ffn
