// Instantiations of fc_tiles (mx4 inputs and weights).
#include "fc_tiles_kernel.h"

namespace cnn {

void run_tiles_mx4(const GroupedFc& p, const TileSize& size, bool vec, float* partial, hipStream_t st) {
    run_tiles<CNN_MX4, CNN_MX4>(p, size, vec, partial, st);
}

}  // namespace cnn
