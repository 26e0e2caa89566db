// Internal declarations of the operators around products on 8-bit floats:
// conversion, the norm, the product and sampling.  No network runs them.
//
// 8-bit floats (CNN_F8): a sign, 4 exponent bits biased by 7, 3 mantissa bits;
// 448 is the largest value, 0x7f and 0xff are NaN, there are no infinities.
// Rows are cut into blocks of 128 values; a scale, fp32, for each.
#pragma once

#include "wide_types.h"

namespace cnn {

constexpr int kF8Block = 128;
constexpr float kF8Most = 448.0f;
constexpr float kF8LeastTop = 0x1p-100f;  // what a block's largest magnitude counts as at least: 448 / it is finite

inline int f8_blocks(int cols) { return ceil_div(cols, kF8Block); }

// Launchers (types: cnn_dtype): arguments already validated.
int launch_f8_quantize(const void* x, int type, int rows, int cols, int block_rows, uint8_t* q, float* scale, hipStream_t st);
int launch_f8_dequantize(const uint8_t* q, const float* scale, int rows, int cols, int block_rows, void* y, int type,
                         hipStream_t st);
// residual, weight, sum: or NULL.  y_type: type, or CNN_F8 with y_scale.
struct RmsNorm {
    const void *x, *residual;
    const float* weight;
    void *sum, *y;
    float* y_scale;
    int type, y_type, rows, cols;
    float eps;
};
int launch_rms_norm(const RmsNorm& p, hipStream_t st);
struct FcF8 {
    const uint8_t* x;
    const float* xs;  // [N][blocks]
    const uint8_t* w;
    const float* ws;  // [ceil(O / 128)][blocks]
    const float* bias;
    void* y;
    int y_type, N, I, O, relu;
};
size_t fc_f8_workspace(int N, int I, int O);
int launch_fc_f8(const FcF8& p, float* ws, hipStream_t st);
struct Sample {
    const void* logits;
    const float *u, *temperature;
    const int32_t* top_k;
    const float *top_p, *min_p;
    int32_t* token;
    float* prob;
    int type, N, V;
};
size_t sample_workspace(int type, int N, int V);
int launch_sample(const Sample& p, void* ws, hipStream_t st);

// 8 values of a row from column c on; columns past the row read as zero.  (The end is
// not computed as c + 8, which for the longest rows is 2^31.)
template <typename T>
__device__ inline void load_values8(const T* row, int c, int cols, float* v) {
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
        for (int i = 0; i < 8; ++i) v[i] = c < cols - i ? to_f32(row[c + i]) : 0.0f;
    }
}
template <typename T>
__device__ inline void store_values8(T* row, int c, int cols, const float* v) {
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
            if (c < cols - i) row[c + i] = from_f32<T>(v[i]);
    }
}

// The largest magnitude of 8 values, as bits that order like it with infinity and NaN on top.
__device__ inline unsigned top_bits8(const float* v) {
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
    return top;
}
// The largest of 16 neighbouring lanes, in all of them: rotations within a row of 16.
__device__ inline unsigned max_of_16_lanes(unsigned v) {
    v = max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x128, 0xf, 0xf, true));  // row_ror 8, 4, 2, 1
    v = max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x124, 0xf, 0xf, true));
    v = max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x122, 0xf, 0xf, true));
    return max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x121, 0xf, 0xf, true));
}

// A block's scale, top / 448, and the factor 448 / top that its values are
// multiplied by, each one rounded division.  A block with an infinity or NaN: NaN and 0.
struct F8Scale {
    float scale, factor;
    bool bad;
    __device__ explicit F8Scale(unsigned top) {
        bad = top >= 0x7f800000u;
        const float a = fmaxf(__uint_as_float(bad ? 0u : top), kF8LeastTop);
        scale = bad ? __uint_as_float(0x7fc00000u) : a / kF8Most;
        factor = kF8Most / a;
    }
};

// 8 values in 8 bits: to the nearest, ties to even.  (A block's largest times its factor is 448 or a rounding more,
// which 448 is the nearest to.)
__device__ inline u32x2 to_f8(const float* v) {
    u32x2 out;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        int w = 0;
        w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h], v[4 * h + 1], w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2], v[4 * h + 3], w, true);
        out[h] = (unsigned)w;
    }
    return out;
}
// ... times the factor, rounded to fp32.
__device__ inline u32x2 to_f8(const float* v, const F8Scale& s) {
    if (s.bad) return u32x2{0, 0};
    float scaled[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) scaled[i] = v[i] * s.factor;
    return to_f8(scaled);
}
__device__ inline void store_f8(uint8_t* row, int c, int cols, u32x2 q) {
    if (c <= cols - 8) {
        __builtin_memcpy(row + c, &q, 8);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c < cols - i) row[c + i] = (uint8_t)(q[i / 4] >> (8 * (i % 4)));
    }
}

}  // namespace cnn
