// Instantiations of fc_tiles (fp32 inputs and weights).
#include "fc_tiles_kernel.h"

namespace cnn {

void run_tiles_f32(const GroupedFc& p, const TileSize& size, bool vec, float* partial, hipStream_t st) {
    run_tiles<CNN_F32, CNN_F32>(p, size, vec, partial, st);
}

}  // namespace cnn
