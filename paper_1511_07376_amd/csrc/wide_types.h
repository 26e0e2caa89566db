// The element types of the operators that take more than fp32, on the device.
#pragma once

#include <hip/hip_runtime.h>

#include "common.h"

namespace cnn {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16_t;
typedef _Float16 f16_t;

inline int type_bytes(int type) { return type == CNN_F32 ? 4 : 2; }

__device__ inline float to_f32(float v) { return v; }
__device__ inline float to_f32(bf16_t v) { return __uint_as_float((unsigned)__builtin_bit_cast(uint16_t, v) << 16); }
__device__ inline float to_f32(f16_t v) { return (float)v; }

// One rounding to the nearest, ties to even.
template <typename T>
__device__ inline T from_f32(float v) {
    return (T)v;
}

// 16 bytes at any address that the elements allow: gfx950 loads and stores
// whole vectors from any byte, and the compiler makes one instruction of this.
template <typename T>
__device__ inline u32x4 load16(const T* p) {
    u32x4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
template <typename T>
__device__ inline void store16(T* p, u32x4 v) {
    __builtin_memcpy(p, &v, 16);
}

// Microscaled 4-bit values: a scale byte s stands for 2^(s - 127), 255 for NaN.
// As the operand of the conversion instructions, which take the exponent
// of a float: 2^-127 is a subnormal one.
__device__ inline float mx4_scale(unsigned s) { return __uint_as_float(s == 0 ? 0x00400000u : s == 255 ? 0x7fc00000u : s << 23); }
constexpr unsigned kMx4NaN = 255;

}  // namespace cnn
