// Instantiations of fc_tiles (bf16 inputs, mx4 weights).
#include "fc_tiles_kernel.h"

namespace cnn {

void run_tiles_wide_mx4(const GroupedFc& p, const TileSize& size, bool vec, float* partial, hipStream_t st) {
    run_tiles<CNN_BF16, CNN_MX4>(p, size, vec, partial, st);
}

}  // namespace cnn
