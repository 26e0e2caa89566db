// Fully connected layers on 8-bit floats with a scale for each block of 128:
//
//     y[n][o] = b[o] + sum_k (xs[n][k] * ws[o / 128][k]) * sum_{i in block k} x[n][i] * w[o][i]
//
// Here: which kernel a call takes, and the one for few tokens.
#include "fc_f8.h"

#include <algorithm>

namespace cnn {
namespace {

constexpr int kMostWaves = 16;

// 16 outputs of 16 NT tokens a workgroup, whose waves share the blocks: the weights are read
// once for all of them, straight to registers.
template <int NT>
__global__ void __launch_bounds__(64 * kMostWaves) fc_f8_rows(FcF8 p, int blocks, int out_groups, int jobs) {
    __shared__ float part[kMostWaves][16 * NT][17];
    const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4;
    const int each = (int)(((int64_t)blocks + waves - 1) / waves);
    const int first = (int)min((int64_t)wave * each, (int64_t)blocks), last = (int)min((int64_t)first + each, (int64_t)blocks);
    const int whole = min(last, p.I / kF8Block);
    for (int job = blockIdx.x; job < jobs; job += gridDim.x) {
        const int o0 = job % out_groups * 16;
        const int64_t n0 = (int64_t)(job / out_groups) * (16 * NT);
        const uint8_t* w = p.w + (size_t)min((int64_t)o0 + l16, (int64_t)p.O - 1) * p.I + quarter * 32;
        const float* ws = p.ws + (size_t)(o0 >> 7) * blocks;
        const uint8_t* x[NT];
        const float* xs[NT];
        f32x4 acc[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int64_t n = min(n0 + 16 * j + l16, (int64_t)p.N - 1);
            x[j] = p.x + (size_t)n * p.I + quarter * 32;
            xs[j] = p.xs + (size_t)n * blocks;
            acc[j] = f32x4{0, 0, 0, 0};
        }
#pragma unroll 2
        for (int k = first; k < whole; ++k) {
            const int64_t at = (int64_t)k * kF8Block;
            const Halves a = to_halves(Bytes{load16(w + at), load16(w + at + 16)});
            const float s = ws[k];
#pragma unroll
            for (int j = 0; j < NT; ++j)
                add_scaled(acc[j], block_sums(a, to_halves(Bytes{load16(x[j] + at), load16(x[j] + at + 16)})), xs[j][k] * s);
        }
        if (whole < last) {
            const int64_t at = (int64_t)whole * kF8Block, in = at + quarter * 32, left = p.I - in;
            auto edge = [&](const uint8_t* row) {
                return to_halves(Bytes{load_bytes_edge(row + at, left, in), load_bytes_edge(row + at + 16, left - 16, in + 16)});
            };
            const Halves a = edge(w);
#pragma unroll
            for (int j = 0; j < NT; ++j) add_scaled(acc[j], block_sums(a, edge(x[j])), xs[j][whole] * ws[whole]);
        }
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[wave][16 * j + l16][quarter * 4 + i] = acc[j][i];
        __syncthreads();
        for (int e = threadIdx.x; e < 256 * NT; e += blockDim.x) {
            const int t = e >> 4, c = e & 15;
            if (n0 + t >= p.N || (int64_t)o0 + c >= p.O) continue;
            float v = 0.0f;
            for (int q = 0; q < waves; ++q) v += part[q][t][c];
            store_value(p.y_type, p.y, (size_t)(n0 + t) * p.O + o0 + c, finish(p, v, p.bias ? p.bias[o0 + c] : 0.0f));
        }
        __syncthreads();
    }
}

template <int NT>
void run_rows(const FcF8& p, hipStream_t st) {
    const int blocks = f8_blocks(p.I), groups = ceil_div(p.O, 16);
    const int64_t jobs = (int64_t)groups * ceil_div(p.N, 16 * NT);
    const int waves = std::max(1, std::min(kMostWaves, blocks / 2));
    enqueue(fc_f8_rows<NT>, dim3((unsigned)std::min<int64_t>(jobs, 1 << 20)), dim3(64 * waves), 0, st, p, blocks, groups, (int)jobs);
}

bool few_rows(const FcF8& p) { return p.N <= 64; }

F8Tile choose_tile(const FcF8& p) {
    const int64_t large = (int64_t)ceil_div(p.O, 256) * ceil_div(p.N, 256);
    if (large >= 192) return {256, 256, 1};
    return {128, 128, 1};
}

}  // namespace

size_t fc_f8_workspace(const FcF8& p) {
    if (p.N == 0 || few_rows(p)) return 0;
    const F8Tile t = choose_tile(p);
    return t.parts > 1 ? (size_t)t.parts * p.N * p.O * sizeof(float) : 0;
}

int launch_fc_f8(const FcF8& p, float* ws, hipStream_t st) {
    if (p.N == 0) return CNN_OK;
    if (few_rows(p)) {
        if (p.N <= 16) run_rows<1>(p, st);
        else if (p.N <= 32) run_rows<2>(p, st);
        else run_rows<4>(p, st);
    } else {
        const bool vec = (uintptr_t)p.x % 16 == 0 && (uintptr_t)p.w % 16 == 0 && p.I % 16 == 0;
        run_f8_tiles(p, choose_tile(p), vec, ws, st);
    }
    return check_launch("fc_f8");
}

}  // namespace cnn
