// Forward products for few rows, fp32 arrays.
#include "ffn_few.h"

namespace ffn {
int launch_few_fp32(const FewArgs& p, int32_t epilogue, int32_t nr, int32_t waves, void* stream) {
    return dev::few<float>(p, epilogue, nr, waves, (hipStream_t)stream);
}
}  // namespace ffn
