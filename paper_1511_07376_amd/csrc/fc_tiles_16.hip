// Instantiations of fc_tiles (bf16 and fp16 inputs and weights).
#include "fc_tiles_kernel.h"

namespace cnn {

void run_tiles_16(const GroupedFc& p, const TileSize& size, bool vec, float* partial, hipStream_t st) {
    if (p.x_type == CNN_BF16) run_tiles<CNN_BF16, CNN_BF16>(p, size, vec, partial, st);
    else run_tiles<CNN_F16, CNN_F16>(p, size, vec, partial, st);
}

}  // namespace cnn
