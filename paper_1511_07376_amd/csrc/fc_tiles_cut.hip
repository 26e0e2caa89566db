// Instantiations of fc_tiles (fp32 and fp16 inputs, mx4 weights).
#include "fc_tiles_kernel.h"

namespace cnn {

void run_tiles_cut(const GroupedFc& p, const TileSize& size, bool vec, float* partial, hipStream_t st) {
    if (p.x_type == CNN_F32) run_tiles<CNN_F32, CNN_MX4>(p, size, vec, partial, st);
    else run_tiles<CNN_F16, CNN_MX4>(p, size, vec, partial, st);
}

}  // namespace cnn
