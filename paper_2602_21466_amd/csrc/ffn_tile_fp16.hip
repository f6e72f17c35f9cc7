// The tiled products for fp16 arrays.
#include "ffn_tile.h"

namespace ffn {
int launch_tile_fp16(const TileArgs& p, int32_t epilogue, bool a_cols, bool b_cols, int32_t tile, void* stream) {
    return dev::run_product<dev::fp16>(p, epilogue, a_cols, b_cols, tile, (hipStream_t)stream);
}
}  // namespace ffn
