// Internal declarations of the operators on microscaled 4-bit values and on
// groups of rows, which no network runs (their kernels and those of the
// networks change apart from each other).
#pragma once

#include "common.h"

namespace cnn {

// Launchers (types: cnn_dtype): arguments already validated.
int launch_mx4_quantize(const void* x, int type, int rows, int cols, uint8_t* q, uint8_t* scale, hipStream_t st);
int launch_mx4_dequantize(const uint8_t* q, const uint8_t* scale, int rows, int cols, void* y, int type, hipStream_t st);
// rows NULL: row m of y is row m of x.  offsets NULL: one group of all M rows.
struct GroupedFc {
    const void* x;
    const uint8_t* xs;  // scales of x, of w: NULL unless mx4
    const int32_t* rows;
    const int32_t* offsets;
    const void* w;
    const uint8_t* ws;
    const float* bias;
    void* y;
    int x_type, w_type, y_type;
    int N, I, M, G, O, relu;
};
// Split reductions leave their sums in the workspace.
size_t fc_grouped_workspace(const GroupedFc& p);
int launch_fc_grouped(const GroupedFc& p, float* ws, hipStream_t st);
size_t route_workspace(int T, int E);
int launch_route(const void* logits, int type, int T, int E, int k, int renorm, int32_t* expert, float* weight,
                 int32_t* rows, int32_t* offsets, int32_t* slot, int32_t* counts, hipStream_t st);
int launch_combine(const void* x, int type, int M, int D, const int32_t* slot, const float* weight, int N, int k,
                   void* y, hipStream_t st);

}  // namespace cnn
