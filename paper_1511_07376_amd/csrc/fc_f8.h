// Products on 8-bit floats by block: operands and sums, for the kernels of fc_f8*.hip.
//
// A block's 128 products of 16 outputs and 16 tokens are summed from zero in fp32 on the
// matrix cores, the scales' product (fp32) multiplies that sum as it is added.  The
// weights are the instructions' first operand and the inputs their second, so that
// a lane's four sums are outputs of one token and share their scale.
//
// A block is summed in 16 bits: every 8-bit float is an fp16 number, the products are exact and are added in
// fp32, at half the 8-bit rate and with conversions.  The 8-bit instructions are no way to do it: they add
// the products of 8 values as fixed-point numbers whose last place is 2^-13 of the power of two at or below the
// largest of them (found by trying, for 16 x 16 x 32, 32 x 32 x 16 and 16 x 16 x 128: random values of all
// exponents come out off by up to 2^-10.3 of the largest product, in 16 bits by 2^-20.9), so that a product
// beside a large one that cancels is lost whole.  What exactness costs: 2048 x 9216 x 4096 to bf16 takes 133 to 146 us
// where it took 77, 512 x 4096 x 4096 28 where it took 18.
#pragma once

#include "f8.h"

namespace cnn {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// 16 bytes of a row from p on of which the first `count` (0 or fewer: none) are in it, zeros behind them;
// `before`: bytes of the row in front.
__device__ inline u32x4 load_bytes_edge(const uint8_t* p, int64_t count, int64_t before) {
    if (count >= 16) return load16(p);
    u32x4 v = {0, 0, 0, 0};
    if (count <= 0) return v;
    const int miss = 16 - (int)count;
    if (before >= miss) {
        const u32x4 last = load16(p - miss);
        const uint64_t lo = last[0] | (uint64_t)last[1] << 32, hi = last[2] | (uint64_t)last[3] << 32;
        const int bits = miss * 8;  // 8 to 120
        const uint64_t l = bits < 64 ? lo >> bits | hi << 1 << (63 - bits) : hi >> (bits - 64), h = bits < 64 ? hi >> bits : 0;
        return u32x4{(unsigned)l, (unsigned)(l >> 32), (unsigned)h, (unsigned)(h >> 32)};
    }
#pragma unroll
    for (int i = 0; i < 15; ++i)
        if (i < count) v[i / 4] |= (unsigned)p[i] << (8 * (i % 4));
    return v;
}

// A lane's 32 values of a block, 16 rows of 4 lanes each: as they are, or as fp16.
struct Bytes {
    u32x4 v[2];
};
// Loads from addresses that are no multiples of 4 take twice as long (300 x 3001 x 1500: 62 us against 28 at 3008).  Such rows
// are loaded by whole words, the first of which can hold bytes from before and the last from behind (the
// same word, so the same page, as one that is wanted), and shifted.
__device__ inline unsigned word_shift(const uint8_t* p) { return (unsigned)(uintptr_t)p & 3; }
__device__ inline u32x4 shifted(u32x4 v, unsigned last, unsigned shift) {
    return u32x4{__builtin_amdgcn_alignbyte(v[1], v[0], shift), __builtin_amdgcn_alignbyte(v[2], v[1], shift),
                 __builtin_amdgcn_alignbyte(v[3], v[2], shift), __builtin_amdgcn_alignbyte(last, v[3], shift)};
}
// 32 bytes from p on.
template <bool ODD>
__device__ inline Bytes load32(const uint8_t* p) {
    if constexpr (!ODD) return Bytes{load16(p), load16(p + 16)};
    const unsigned shift = word_shift(p);
    const uint8_t* words = p - shift;
    const u32x4 a = load16(words), b = load16(words + 16);
    unsigned last;
    __builtin_memcpy(&last, words + (shift ? 32 : 28), 4);
    return Bytes{shifted(a, b[0], shift), shifted(b, last, shift)};
}
struct Halves {
    f16x8 v[4];
};
__device__ inline f16x8 to_halves(unsigned a, unsigned b) {
    const f16x2 p = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)a, 1.0f, false), q = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)a, 1.0f, true);
    const f16x2 r = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)b, 1.0f, false), s = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)b, 1.0f, true);
    return f16x8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}
__device__ inline Halves to_halves(const Bytes& b) {
    return Halves{to_halves(b.v[0][0], b.v[0][1]), to_halves(b.v[0][2], b.v[0][3]), to_halves(b.v[1][0], b.v[1][1]), to_halves(b.v[1][2], b.v[1][3])};
}

// A block's sums: output 4 (lane / 16) + i of token lane % 16.
__device__ inline f32x4 block_sums(const Halves& w, const Halves& x) {
    f32x4 d = {0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < 4; ++c) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(w.v[c], x.v[c], d, 0, 0, 0);
    return d;
}
__device__ inline void add_scaled(f32x4& acc, f32x4 d, float s) {
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = fmaf(s, d[i], acc[i]);
}

__device__ inline float finish(const FcF8& p, float v, float bias) {
    v += bias;
    return p.relu ? (v > 0.0f ? v : 0.0f) : v;
}
__device__ inline void store_value(int type, void* y, size_t at, float v) {
    if (type == CNN_F32) ((float*)y)[at] = v;
    else if (type == CNN_BF16) ((bf16_t*)y)[at] = from_f32<bf16_t>(v);
    else ((f16_t*)y)[at] = from_f32<f16_t>(v);
}

// A tile's size, and the parts its reduction is split into (over workgroups, joined by a second
// kernel), of `run` blocks each, a multiple of 4.
struct F8Tile {
    int outs, tokens, parts, run;
};
// Which kernel a product takes: by rows, 16 times `tokens` of them and 16 times `outs` outputs a workgroup, or on a tile.
struct F8Way {
    int rows, tokens, outs;
    F8Tile tile;
};
F8Way fc_f8_way(int N, int I, int O);
// vec: rows of whole blocks at 16-byte addresses.
void run_f8_tiles(const FcF8& p, const F8Tile& tile, bool vec, float* partial, hipStream_t st);

}  // namespace cnn
