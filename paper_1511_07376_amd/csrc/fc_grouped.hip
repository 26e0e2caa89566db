// Fully connected layers whose rows belong to groups with weights of their own
// (one group: a plain layer), and whose operands may be narrower than fp32:
//
//     y[m][o] = b[g][o] + sum_i x[rows[m]][i] * w[g][o][i],  offsets[g] <= m < offsets[g + 1]
//
// Sums are held in fp32 and rounded once, to the type of y.
#include "fc_operands.h"

#include <algorithm>

namespace cnn {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

// Tile t of the launch: tiles of TM rows, numbered through the groups.  False
// behind the last one.  The wave looks at 64 groups at a time; the answer is
// uniform.
template <int TM>
__device__ inline bool find_tile(const GroupedFc& p, int64_t t, int& g, int& row0, int& hi) {
    if (!p.offsets) {
        g = 0;
        row0 = (int)(t * TM);
        hi = p.M;
        return t * TM < p.M;
    }
    const int lane = threadIdx.x & 63;
    int64_t before = 0;
    for (int base = 0; base < p.G; base += 64) {
        int lo = 0, end = 0;
        if (base + lane < p.G) group_rows(p.offsets, base + lane, p.M, lo, end);
        const int tiles = (int)(((unsigned)(end - lo) + TM - 1) / TM);
        int incl = tiles;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int u = __shfl_up(incl, off);
            if (lane >= off) incl += u;
        }
        const unsigned long long past = __ballot(before + incl > t);
        if (past) {
            const int at = __builtin_ctzll(past);
            g = __builtin_amdgcn_readfirstlane(base + at);
            const int first = (int)(t - before) - (__shfl(incl, at) - __shfl(tiles, at));
            row0 = __builtin_amdgcn_readfirstlane(__shfl(lo, at) + first * TM);
            hi = __builtin_amdgcn_readfirstlane(__shfl(end, at));
            return true;
        }
        before += __shfl(incl, 63);
    }
    return false;
}

__device__ inline float element(const void* base, int type, size_t i) {
    if (type == CNN_F32) return ((const float*)base)[i];
    if (type == CNN_BF16) return to_f32(((const bf16_t*)base)[i]);
    return to_f32(((const f16_t*)base)[i]);
}

// Element c of a row of mx4 blocks.
__device__ inline float element_mx4(const uint8_t* row, const uint8_t* scale, int c) {
    const unsigned byte = row[c >> 1];
    const unsigned s = scale[c >> 5];
    const float f = mx4_scale(s);
    const f32x2 v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(byte, f, 0);
    return s == kMx4NaN ? f : v[c & 1];
}

__device__ inline void store_element(void* base, int type, size_t i, float v) {
    if (type == CNN_F32) ((float*)base)[i] = v;
    else if (type == CNN_BF16) ((bf16_t*)base)[i] = from_f32<bf16_t>(v);
    else ((f16_t*)base)[i] = from_f32<f16_t>(v);
}

constexpr int kTile = 16;

__global__ void __launch_bounds__(kTile * kTile) fc_grouped_plain(GroupedFc p, int64_t tiles, int cols) {
    __shared__ float sx[kTile][kTile + 1], sw[kTile][kTile + 1];
    const int a = threadIdx.x % kTile, b = threadIdx.x / kTile;
    const int64_t blocks = (p.I + 31) / 32;
    for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
        int g, row0, hi;
        if (!find_tile<kTile>(p, t / cols, g, row0, hi)) break;
        const int o0 = (int)(t % cols) * kTile;
        const int m = row0 + b, o = o0 + a;
        int src = m < hi ? (p.rows ? p.rows[m] : m) : -1;
        if (src >= p.N) src = -1;
        const int wrow = min(o0 + b, p.O - 1);
        const size_t wat = (size_t)g * p.O + wrow;
        float acc = 0.0f;
        for (int k0 = 0; k0 < p.I; k0 += kTile) {
            const int c = k0 + a;
            float xv = 0.0f, wv = 0.0f;
            if (c < p.I) {
                if (src >= 0)
                    xv = p.x_type == CNN_MX4 ? element_mx4((const uint8_t*)p.x + (size_t)src * blocks * 16, p.xs + (size_t)src * blocks, c)
                                             : element(p.x, p.x_type, (size_t)src * p.I + c);
                wv = p.w_type == CNN_MX4 ? element_mx4((const uint8_t*)p.w + wat * blocks * 16, p.ws + wat * blocks, c)
                                         : element(p.w, p.w_type, wat * p.I + c);
            }
            sx[b][a] = xv;
            sw[b][a] = wv;
            __syncthreads();
            for (int i = 0; i < kTile; ++i) acc = fmaf(sx[b][i], sw[a][i], acc);
            __syncthreads();
        }
        if (m < hi && o < p.O) {
            if (src < 0) acc = 0.0f;
            if (p.bias) acc += p.bias[(size_t)g * p.O + o];
            if (p.relu) acc = acc > 0.0f ? acc : 0.0f;
            store_element(p.y, p.y_type, (size_t)m * p.O + o, acc);
        }
    }
}

}  // namespace

int launch_fc_grouped(const GroupedFc& p, hipStream_t st) {
    if (p.M == 0) return CNN_OK;
    if (ceil_div64(p.M, p.G) <= 32) return run_fc_rows(p, st);
    const int64_t row_tiles = ceil_div64(p.M, kTile) + (p.offsets ? p.G : 0);
    const int cols = ceil_div(p.O, kTile);
    const int64_t tiles = row_tiles * cols;
    enqueue(fc_grouped_plain, dim3((unsigned)std::min<int64_t>(tiles, 1 << 20)), dim3(kTile * kTile), 0, st, p, tiles, cols);
    return check_launch("fc_grouped");
}

}  // namespace cnn
