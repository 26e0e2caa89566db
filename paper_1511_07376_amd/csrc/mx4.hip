// Microscaled 4-bit values (mx4): a row is cut into blocks of 32, a block is 16
// bytes of 4-bit values (sign, 2 exponent bits, 1 mantissa bit: 0, 0.5, 1,
// 1.5, 2, 3, 4, 6) and one byte s that scales them by 2^(s - 127).
//
// To mx4: with a the largest magnitude of the block, s - 127 =
// floor(log2 a) - 2, so that a lies in [4, 8) times the scale, where 6 is the
// largest value; every element is divided by the scale and rounded to
// the nearest value, ties to the even code, and what is above 6 becomes 6.
// floor(log2 a) is the exponent field of a as a float, so the maximum is
// taken over the bit patterns of the magnitudes, which order as the numbers
// do and put NaN and infinity above all of them: a block that holds
// one gets s = 255 and reads as NaN.
//
// Both directions move bytes and little else (HBM bound).  A work-item takes 8
// values, a quarter of a block: 16 or 32 bytes of wide values against 4 of
// 4-bit ones, the conversion instructions of gfx950 in between.  fp32 4096 x 9216:
// 36.2 us to mx4 and 28.3 back (4.7 and 6.0 TB/s, some of them from the memory-side
// cache), bf16 64 x 4096: 2.6 and 2.5 (a kernel's least).
#include "experts.h"
#include "wide_types.h"

#include <algorithm>

namespace cnn {
namespace {

constexpr int kThreads = 256;

typedef float f32x2 __attribute__((ext_vector_type(2)));

// 8 values of a row from column c on; columns past the row read as zero.  (The end is
// not computed as c + 8, which for the longest rows is 2^31.)
template <typename T>
__device__ inline void load8(const T* row, int c, int cols, float* v) {
    if (c <= cols - 8) {
        constexpr int N = 16 / (int)sizeof(T);
#pragma unroll
        for (int h = 0; h < 8 / N; ++h) {
            T part[N];
            const u32x4 u = load16(row + c + h * N);
            __builtin_memcpy(part, &u, 16);
#pragma unroll
            for (int i = 0; i < N; ++i) v[h * N + i] = to_f32(part[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? to_f32(row[c + i]) : 0.0f;
    }
}

template <typename T>
__device__ inline void store8(T* row, int c, int cols, const float* v) {
    if (c <= cols - 8) {
        constexpr int N = 16 / (int)sizeof(T);
#pragma unroll
        for (int h = 0; h < 8 / N; ++h) {
            T part[N];
#pragma unroll
            for (int i = 0; i < N; ++i) part[i] = from_f32<T>(v[h * N + i]);
            u32x4 u;
            __builtin_memcpy(&u, part, 16);
            store16(row + c + h * N, u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) row[c + i] = from_f32<T>(v[i]);
    }
}

// Item 4 u + j is quarter j of block u; blocks are numbered through the rows.
template <typename T>
__global__ void __launch_bounds__(kThreads)
mx4_quantize(const T* x, uint8_t* q, uint8_t* scale, int64_t items, int cols, FastDiv f_blocks, int blocks) {
    const int64_t step = (int64_t)gridDim.x * kThreads;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < items; i += step) {
        const unsigned u = (unsigned)(i >> 2);
        const int row = (int)fdiv(u, f_blocks);
        const int c = ((int)u - row * blocks) * 32 + ((int)i & 3) * 8;
        float v[8];
        load8(x + (size_t)row * cols, c, cols, v);
        unsigned top = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint(v[k]) & 0x7fffffffu);
        // the four work-items of a block are neighbours, and all or none are here
        top = max(top, (unsigned)__shfl_xor((int)top, 1));
        top = max(top, (unsigned)__shfl_xor((int)top, 2));
        const unsigned e = top >> 23;
        const unsigned s = e == kMx4NaN ? kMx4NaN : e > 2 ? e - 2 : 0;
        unsigned out = 0;
        if (s != kMx4NaN) {
            const float f = mx4_scale(s);
            out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, v[0], v[1], f, 0);
            out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, v[2], v[3], f, 1);
            out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, v[4], v[5], f, 2);
            out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, v[6], v[7], f, 3);
        }
        __builtin_memcpy(q + i * 4, &out, 4);
        if ((i & 3) == 0) scale[u] = (uint8_t)s;
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
mx4_dequantize(const uint8_t* q, const uint8_t* scale, T* y, int64_t items, int cols, FastDiv f_blocks, int blocks) {
    const int64_t step = (int64_t)gridDim.x * kThreads;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < items; i += step) {
        const unsigned u = (unsigned)(i >> 2);
        const int row = (int)fdiv(u, f_blocks);
        const int c = ((int)u - row * blocks) * 32 + ((int)i & 3) * 8;
        unsigned in;
        __builtin_memcpy(&in, q + i * 4, 4);
        const unsigned s = scale[u];
        const float f = mx4_scale(s);
        float v[8];
#define CNN_PAIR(k)                                                             \
    {                                                                           \
        const f32x2 p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in, f, k);     \
        v[2 * k] = p[0];                                                        \
        v[2 * k + 1] = p[1];                                                    \
    }
        CNN_PAIR(0) CNN_PAIR(1) CNN_PAIR(2) CNN_PAIR(3)
#undef CNN_PAIR
        if (s == kMx4NaN) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = f;
        }
        store8(y + (size_t)row * cols, c, cols, v);
    }
}

dim3 grid_for(int64_t items) {
    return dim3((unsigned)std::min<int64_t>(ceil_div64(items, kThreads), 1 << 20));
}

}  // namespace

int launch_mx4_quantize(const void* x, int type, int rows, int cols, uint8_t* q, uint8_t* scale, hipStream_t st) {
    const int blocks = ceil_div(cols, 32);
    const int64_t items = (int64_t)rows * blocks * 4;
    if (items == 0) return CNN_OK;
    const FastDiv f = make_fastdiv(blocks);
    if (type == CNN_F32)
        enqueue(mx4_quantize<float>, grid_for(items), dim3(kThreads), 0, st, (const float*)x, q, scale, items, cols, f, blocks);
    else if (type == CNN_BF16)
        enqueue(mx4_quantize<bf16_t>, grid_for(items), dim3(kThreads), 0, st, (const bf16_t*)x, q, scale, items, cols, f, blocks);
    else
        enqueue(mx4_quantize<f16_t>, grid_for(items), dim3(kThreads), 0, st, (const f16_t*)x, q, scale, items, cols, f, blocks);
    return check_launch("mx4_quantize");
}

int launch_mx4_dequantize(const uint8_t* q, const uint8_t* scale, int rows, int cols, void* y, int type, hipStream_t st) {
    const int blocks = ceil_div(cols, 32);
    const int64_t items = (int64_t)rows * blocks * 4;
    if (items == 0) return CNN_OK;
    const FastDiv f = make_fastdiv(blocks);
    if (type == CNN_F32)
        enqueue(mx4_dequantize<float>, grid_for(items), dim3(kThreads), 0, st, q, scale, (float*)y, items, cols, f, blocks);
    else if (type == CNN_BF16)
        enqueue(mx4_dequantize<bf16_t>, grid_for(items), dim3(kThreads), 0, st, q, scale, (bf16_t*)y, items, cols, f, blocks);
    else
        enqueue(mx4_dequantize<f16_t>, grid_for(items), dim3(kThreads), 0, st, q, scale, (f16_t*)y, items, cols, f, blocks);
    return check_launch("mx4_dequantize");
}

}  // namespace cnn
