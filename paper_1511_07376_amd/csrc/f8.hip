// Rows of wide values to 8-bit floats and back, a scale for each block of 128
// values of a row (activations) or of 128 rows of 128 (weights).
//
// With a the largest magnitude of a block (2^-100 at least): scale = a / 448, and every
// value times 448 / a, rounded to the nearest 8-bit float.  The maximum is taken
// over the bit patterns of the magnitudes, which order as the numbers do and put
// infinity and NaN above all of them: such a block gets NaN for its scale.
//
// Both directions move bytes and little else (HBM bound).  A work-item takes 8
// values, so that 16 lanes are a block of a row, whose maximum four moves between lanes find.  4096 x 9216
// fp32: rows 34 us (5.6 TB/s, above a copy's 5.05, as it mostly reads), squares 37 us (5.1), back 37 us
// (5.1); bf16 23, 30 and 22 us; 64 x 4096 2.7 us, the least of a kernel.
#include "f8.h"

#include <algorithm>

namespace cnn {
namespace {

constexpr int kThreads = 256;

typedef float f32x2 __attribute__((ext_vector_type(2)));

// Item 16 u + j is the 8 values j of block u; blocks are numbered through the rows.
template <typename T>
__global__ void __launch_bounds__(kThreads)
f8_quantize_rows(const T* x, uint8_t* q, float* scale, int64_t items, int cols, FastDiv f_blocks, int blocks) {
    const int64_t step = (int64_t)gridDim.x * kThreads;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < items; i += step) {
        const unsigned u = (unsigned)(i >> 4);
        const int row = (int)fdiv(u, f_blocks);
        const int64_t at = (int64_t)((int)u - row * blocks) * kF8Block + ((int)i & 15) * 8;
        const int c = at < cols ? (int)at : cols;
        float v[8];
        load_values8(x + (size_t)row * cols, c, cols, v);
        // the 16 work-items of a block are neighbours, and all or none are here
        const F8Scale s(max_of_16_lanes(top_bits8(v)));
        store_f8(q + (size_t)row * cols, c, cols, to_f8(v, s));
        if ((i & 15) == 0) scale[u] = s.scale;
    }
}

// A workgroup takes 128 rows of 128 values: 16 rows at a time, 8 times, held in registers.  (Weights are laid out
// once: 16384 x 1013 bf16, whose rows begin at any element, takes 22 us against 12.5 by rows.)
template <typename T>
__global__ void __launch_bounds__(kThreads)
f8_quantize_squares(const T* x, uint8_t* q, float* scale, int rows, int cols, int blocks, int64_t squares) {
    __shared__ unsigned sTop[kThreads / 64];
    const int tid = threadIdx.x;
    for (int64_t b = blockIdx.x; b < squares; b += gridDim.x) {
        const int64_t r0 = b / blocks * kF8Block;
        const int64_t at = b % blocks * kF8Block + (tid & 15) * 8;
        const int c = at < cols ? (int)at : cols;
        float v[8][8];
        unsigned top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t r = r0 + j * 16 + (tid >> 4);
            load_values8(x + (size_t)min(r, (int64_t)rows - 1) * cols, c, r < rows ? cols : 0, v[j]);
            top = max(top, top_bits8(v[j]));
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, off));
        __syncthreads();  // the last square's maxima have been read
        if ((tid & 63) == 0) sTop[tid >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) top = max(top, sTop[w]);
        const F8Scale s(top);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t r = r0 + j * 16 + (tid >> 4);
            if (r < rows) store_f8(q + (size_t)r * cols, c, cols, to_f8(v[j], s));
        }
        if (tid == 0) scale[b] = s.scale;
    }
}

// Item j of a row is its values from 8 j on.
template <typename T>
__global__ void __launch_bounds__(kThreads)
f8_dequantize(const uint8_t* q, const float* scale, T* y, int64_t items, int cols, FastDiv f_each, int each, int blocks, int row_shift) {
    const int64_t step = (int64_t)gridDim.x * kThreads;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < items; i += step) {
        const int row = (int)fdiv((unsigned)i, f_each);
        const int c = ((int)i - row * each) * 8;
        const uint8_t* src = q + (size_t)row * cols;
        u32x2 in = {0, 0};
        if (c <= cols - 8) {
            __builtin_memcpy(&in, src + c, 8);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c < cols - k) in[k / 4] |= (unsigned)src[c + k] << (8 * (k % 4));
        }
        const float f = scale[(size_t)(row >> row_shift) * blocks + c / kF8Block];
        float v[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)in[h], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)in[h], true);
            v[4 * h] = a[0] * f;
            v[4 * h + 1] = a[1] * f;
            v[4 * h + 2] = b[0] * f;
            v[4 * h + 3] = b[1] * f;
        }
        store_values8(y + (size_t)row * cols, c, cols, v);
    }
}

dim3 grid_for(int64_t items) { return dim3((unsigned)std::min<int64_t>(ceil_div64(items, kThreads), 1 << 20)); }

template <typename T>
void quantize(const void* x, int rows, int cols, int block_rows, uint8_t* q, float* scale, hipStream_t st) {
    const int blocks = f8_blocks(cols);
    if (block_rows == 1) {
        const int64_t items = (int64_t)rows * blocks * 16;
        enqueue(f8_quantize_rows<T>, grid_for(items), dim3(kThreads), 0, st, (const T*)x, q, scale, items, cols, make_fastdiv(blocks), blocks);
    } else {
        const int64_t squares = ceil_div64(rows, kF8Block) * blocks;
        enqueue(f8_quantize_squares<T>, dim3((unsigned)std::min<int64_t>(squares, 1 << 20)), dim3(kThreads), 0, st, (const T*)x, q, scale, rows, cols, blocks, squares);
    }
}

template <typename T>
void dequantize(const uint8_t* q, const float* scale, int rows, int cols, int block_rows, void* y, hipStream_t st) {
    const int each = ceil_div(cols, 8);
    const int64_t items = (int64_t)rows * each;
    enqueue(f8_dequantize<T>, grid_for(items), dim3(kThreads), 0, st, q, scale, (T*)y, items, cols, make_fastdiv(each), each, f8_blocks(cols), block_rows == 1 ? 0 : 7);
}

}  // namespace

int launch_f8_quantize(const void* x, int type, int rows, int cols, int block_rows, uint8_t* q, float* scale, hipStream_t st) {
    if (rows == 0) return CNN_OK;
    if (type == CNN_F32) quantize<float>(x, rows, cols, block_rows, q, scale, st);
    else if (type == CNN_BF16) quantize<bf16_t>(x, rows, cols, block_rows, q, scale, st);
    else quantize<f16_t>(x, rows, cols, block_rows, q, scale, st);
    return check_launch("f8_quantize");
}

int launch_f8_dequantize(const uint8_t* q, const float* scale, int rows, int cols, int block_rows, void* y, int type,
                         hipStream_t st) {
    if (rows == 0) return CNN_OK;
    if (type == CNN_F32) dequantize<float>(q, scale, rows, cols, block_rows, y, st);
    else if (type == CNN_BF16) dequantize<bf16_t>(q, scale, rows, cols, block_rows, y, st);
    else dequantize<f16_t>(q, scale, rows, cols, block_rows, y, st);
    return check_launch("f8_dequantize");
}

}  // namespace cnn
