// Operands of the products on groups of rows, as the matrix cores take them.
//
// A lane feeds the matrix cores runs of 32 consecutive values of a row (an mx4
// block, 64 bytes of a 16-bit type, 128 of fp32).  Which k of the
// reduction an instruction's slot stands for is free as long as both operands
// agree, so a run is cut into the instruction's lane parts in order: 4 of 8
// values for the 16-bit instructions, 32 single ones for the fp32 one, and
// whole for the scaled 4-bit one.
//
// Wide inputs with mx4 weights: the weights' values (2 significant bits and
// a power of two) are bfloat16 numbers, and so are the parts that a wider
// input is cut into: its leading 8 bits, the next 8, the rest (one part for
// bf16, two for fp16, three for fp32).  Every product is then exact in the
// fp32 sums.
#pragma once

#include "experts.h"
#include "wide_types.h"

#include <cmath>

namespace cnn {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// Bytes of a run of 32 values, and its 16-byte loads.
template <int T>
constexpr int kRunBytes = T == CNN_F32 ? 128 : T == CNN_MX4 ? 16 : 64;
template <int T>
constexpr int kRunLoads = kRunBytes<T> / 16;
template <int T>
constexpr int kElemBytes = T == CNN_F32 ? 4 : 2;  // wide types

// Parts that an input of type XT is cut into beside mx4 weights.
template <int XT>
constexpr int kParts = XT == CNN_F32 ? 3 : XT == CNN_F16 ? 2 : 1;

// A 16-byte vector of which the first `count` values are in a row (0 or
// fewer: none), zeros behind them; `before`: values of the row in front of it.  One
// load, of the row's last 16 bytes, and a shift; a row shorter than
// that is taken value by value.
template <int T>
__device__ inline u32x4 load_vector_edge(const char* p, int count, int64_t before) {
    constexpr int ES = kElemBytes<T>, N = 16 / ES;
    if (count >= N) return load16(p);
    u32x4 v = {0, 0, 0, 0};
    if (count <= 0) return v;
    if (before >= N - count) {
        const u32x4 last = load16(p - (N - count) * ES);
        const uint64_t lo = last[0] | (uint64_t)last[1] << 32, hi = last[2] | (uint64_t)last[3] << 32;
        const int bits = (N - count) * ES * 8;  // of 2 to 14 bytes
        const uint64_t l = bits < 64 ? lo >> bits | hi << 1 << (63 - bits) : hi >> (bits - 64), h = bits < 64 ? hi >> bits : 0;
        return u32x4{(unsigned)l, (unsigned)(l >> 32), (unsigned)h, (unsigned)(h >> 32)};
    }
#pragma unroll
    for (int c = 0; c < N; ++c) {
        if (c < count) {
            if constexpr (ES == 4) {
                unsigned e;
                __builtin_memcpy(&e, p + c * 4, 4);
                v[c] = e;
            } else {
                uint16_t e;
                __builtin_memcpy(&e, p + c * 2, 2);
                v[c / 2] |= (unsigned)e << (16 * (c % 2));
            }
        }
    }
    return v;
}

// `count` values (0 or fewer: none) from p on in 16-byte vectors, zeros behind them.
template <int T, int LOADS>
__device__ inline void load_edge(const char* p, int count, int64_t before, u32x4* v) {
    constexpr int N = 16 / kElemBytes<T>;
#pragma unroll
    for (int h = 0; h < LOADS; ++h) v[h] = load_vector_edge<T>(p + h * 16, count - h * N, before + h * N);
}

// 32 values of a row that ends after `cols` of them, from k on; past the end
// they are 0.  FULL: all are inside.  ODD: the row's address may be no multiple of 4,
// which makes loads of 16-bit values 2 to 3 times as long (88 rows to 24 groups
// of 2101 x 1387, fp16: 84 us; of 2104 x 1387 36).  Then whole words are
// loaded, the first of which can hold a value from before the row and the last one
// from behind it, and straighten_run() shifts them once they are there.
template <int T, bool FULL, bool ODD>
__device__ inline void load_run(const char* row, int64_t k, int cols, u32x4* run, unsigned& last) {
    constexpr int ES = kElemBytes<T>;
    if constexpr (FULL && ODD && ES == 2) {
        const int shift = (int)((uintptr_t)row & 2);
        const char* words = row + k * ES - shift;
#pragma unroll
        for (int j = 0; j < kRunLoads<T>; ++j) run[j] = load16(words + j * 16);
        __builtin_memcpy(&last, words + (shift ? 64 : 60), 4);
    } else if (FULL || k + 32 <= cols) {
#pragma unroll
        for (int j = 0; j < kRunLoads<T>; ++j) run[j] = load16(row + k * ES + j * 16);
    } else {
        load_edge<T, kRunLoads<T>>(row + k * ES, (int)max((int64_t)cols - k, (int64_t)0), k, run);
    }
}
template <int T, bool FULL, bool ODD>
__device__ inline void straighten_run(const char* row, u32x4* run, unsigned last) {
    if constexpr (FULL && ODD && kElemBytes<T> == 2) {
        const unsigned bits = (unsigned)((uintptr_t)row & 2) * 8;
#pragma unroll
        for (int c = 0; c < 16; ++c)
            run[c / 4][c % 4] = __builtin_amdgcn_alignbit(c < 15 ? run[(c + 1) / 4][(c + 1) % 4] : last, run[c / 4][c % 4], bits);
    }
}

// The leading bfloat16 of each of two floats, cut and not rounded (so that the
// largest stay finite), packed; the floats become what it leaves.  Exact: a
// float has 24 bits, its leading part takes 8 and leaves 16 or fewer.  NaN
// leaves NaN.  Infinity leaves NaN too, and 0 with SAFE, which costs four
// more instructions.
template <bool SAFE>
__device__ inline unsigned cut_pair(float& a, float& b) {
    const unsigned ua = __float_as_uint(a), ub = __float_as_uint(b);
    const unsigned packed = __builtin_amdgcn_perm(ub, ua, 0x07060302u);
    const float ra = a - __uint_as_float(ua & 0xffff0000u), rb = b - __uint_as_float(ub & 0xffff0000u);
    a = SAFE && __builtin_isinf(a) ? 0.0f : ra;
    b = SAFE && __builtin_isinf(b) ? 0.0f : rb;
    return packed;
}

template <int PARTS, bool SAFE>
__device__ inline void cut8(float* v, u32x4* part) {
#pragma unroll
    for (int q = 0; q < PARTS; ++q)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if (q + 1 < PARTS)
                part[q][c] = cut_pair<SAFE>(v[2 * c], v[2 * c + 1]);
            else  // what is left has 8 bits at most (below 2^-107: is cut at 2^-133)
                part[q][c] = __builtin_amdgcn_perm(__float_as_uint(v[2 * c + 1]), __float_as_uint(v[2 * c]), 0x07060302u);
        }
}

// 8 values of wide type XT (at `run`, 16 or 32 bytes) as bfloat16 parts.
template <int XT>
__device__ inline void cut_parts(const u32x4* run, u32x4* part) {
    if constexpr (XT == CNN_BF16) {
        part[0] = run[0];
    } else {
        float v[8], top = 0.0f;
        if constexpr (XT == CNN_F16) {
            const f16x8 h = __builtin_bit_cast(f16x8, run[0]);
#pragma unroll
            for (int c = 0; c < 8; ++c) v[c] = (float)h[c];
        } else {
#pragma unroll
            for (int c = 0; c < 8; ++c) v[c] = __uint_as_float(run[c / 4][c % 4]);
        }
        // infinities are rare: one test for eight values, and the wave's lanes together
#pragma unroll
        for (int c = 0; c < 8; ++c) top = fmaxf(top, fabsf(v[c]));
        if (__any(top == INFINITY)) cut8<kParts<XT>, true>(v, part);
        else cut8<kParts<XT>, false>(v, part);
    }
}

// 8 values of an mx4 block (word j) as bfloat16.
__device__ inline bf16x8 decode8(unsigned word, float scale) {
    u32x4 out;
    out[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 0));
    out[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 1));
    out[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 2));
    out[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 3));
    return __builtin_bit_cast(bf16x8, out);
}

__device__ inline i32x8 mx4_operand(u32x4 v) { return i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0}; }

// The rows of a group, clipped to [0, M): offsets are the caller's data.
__device__ inline void group_rows(const int32_t* offsets, int g, int M, int& lo, int& hi) {
    lo = min(max(offsets[g], 0), M);
    hi = min(max(offsets[g + 1], lo), M);
}

// The row of x that row m of y is made of; < 0 where there is none.
__device__ inline int source_row(const GroupedFc& p, int m) {
    const int r = p.rows ? p.rows[m] : m;
    return r < p.N ? r : -1;
}

template <int YT>
__device__ inline void store_result(void* y, size_t i, float v) {
    if constexpr (YT == CNN_F32) ((float*)y)[i] = v;
    else if constexpr (YT == CNN_BF16) ((bf16_t*)y)[i] = from_f32<bf16_t>(v);
    else ((f16_t*)y)[i] = from_f32<f16_t>(v);
}
__device__ inline void store_result(int type, void* y, size_t i, float v) {
    if (type == CNN_F32) store_result<CNN_F32>(y, i, v);
    else if (type == CNN_BF16) store_result<CNN_BF16>(y, i, v);
    else store_result<CNN_F16>(y, i, v);
}

int run_fc_rows(const GroupedFc& p, hipStream_t st);

}  // namespace cnn
