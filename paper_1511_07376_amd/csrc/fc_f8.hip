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

// 16 FO outputs of 16 NT tokens a workgroup, whose waves share the blocks: the weights are read
// once for all of them, straight to registers, and the waves' sums are joined in LDS, in their order.  Bound by
// reading: 1 x 9216 x 8192 takes 14.5 us (5.2 TB/s), 1 x 4096 x 4096 5 to 7 (a chain of load, product and
// join), 77 x 1013 x 610, whose rows begin at any byte, 5.4 to 6.6.
template <int NT, int FO, bool ODD>
__global__ void __launch_bounds__(64 * kMostWaves) fc_f8_rows(FcF8 p, int blocks, int out_groups, int jobs) {
    __shared__ float part[kMostWaves][16 * NT][16 * FO + 1];
    const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4;
    const int each = (int)(((int64_t)blocks + waves - 1) / waves);
    const int first = (int)min((int64_t)wave * each, (int64_t)blocks), last = (int)min((int64_t)first + each, (int64_t)blocks);
    const int whole = min(last, p.I / kF8Block);
    for (int job = blockIdx.x; job < jobs; job += gridDim.x) {
        const int o0 = job % out_groups * (16 * FO);
        const int64_t n0 = (int64_t)(job / out_groups) * (16 * NT);
        const float* ws = p.ws + (size_t)(o0 >> 7) * blocks;
        // (offsets of 32 bits: a tensor has fewer than 2^31 bytes)
        unsigned w[FO], x[NT], xs[NT];
        f32x4 acc[FO][NT];
#pragma unroll
        for (int i = 0; i < FO; ++i) w[i] = (unsigned)min((int64_t)o0 + 16 * i + l16, (int64_t)p.O - 1) * (unsigned)p.I + quarter * 32;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const unsigned n = (unsigned)min(n0 + 16 * j + l16, (int64_t)p.N - 1);
            x[j] = n * (unsigned)p.I + quarter * 32;
            xs[j] = n * (unsigned)blocks;
#pragma unroll
            for (int i = 0; i < FO; ++i) acc[i][j] = f32x4{0, 0, 0, 0};
        }
        auto add = [&](int k, auto&& load) {
            Halves a[FO];
            Bytes raw[FO], b[NT];
            float s[NT];
#pragma unroll
            for (int i = 0; i < FO; ++i) raw[i] = load(p.w, w[i]);
#pragma unroll
            for (int j = 0; j < NT; ++j) b[j] = load(p.x, x[j]), s[j] = (p.xs + k)[xs[j]] * ws[k];
#pragma unroll
            for (int i = 0; i < FO; ++i) a[i] = to_halves(raw[i]);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const Halves h = to_halves(b[j]);
#pragma unroll
                for (int i = 0; i < FO; ++i) add_scaled(acc[i][j], block_sums(a[i], h), s[j]);
            }
        };
        for (int k = first; k < whole; ++k) {
            const int64_t at = (int64_t)k * kF8Block;
            add(k, [&](const uint8_t* base, unsigned row) { return load32<ODD>(base + at + row); });
        }
        if (first < last && whole < last) {  // (waves behind the last block have none)
            const int64_t at = (int64_t)whole * kF8Block, in = at + quarter * 32, left = p.I - in;
            add(whole, [&](const uint8_t* base, unsigned row) {
                return Bytes{load_bytes_edge(base + at + row, left, in), load_bytes_edge(base + at + row + 16, left - 16, in + 16)};
            });
        }
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < FO; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) part[wave][16 * j + l16][16 * i + quarter * 4 + c] = acc[i][j][c];
        __syncthreads();
        for (int e = threadIdx.x; e < 256 * NT * FO; e += blockDim.x) {
            const int t = e / (16 * FO), c = e % (16 * FO);
            if (n0 + t >= p.N || (int64_t)o0 + c >= p.O) continue;
            float v = 0.0f;
            for (int q = 0; q < waves; ++q) v += part[q][t][c];
            store_value(p.y_type, p.y, (size_t)(n0 + t) * p.O + o0 + c, finish(p, v, p.bias ? p.bias[o0 + c] : 0.0f));
        }
        __syncthreads();
    }
}

template <int NT, int FO>
void run_rows(const FcF8& p, bool odd, hipStream_t st) {
    const int blocks = f8_blocks(p.I), groups = ceil_div(p.O, 16 * FO);
    const int64_t jobs = (int64_t)groups * ceil_div(p.N, 16 * NT);
    const int waves = std::max(1, std::min(kMostWaves, blocks / 2));
    const dim3 grid((unsigned)std::min<int64_t>(jobs, 1 << 20)), block(64 * waves);
    if (odd) enqueue(fc_f8_rows<NT, FO, true>, grid, block, 0, st, p, blocks, groups, (int)jobs);
    else enqueue(fc_f8_rows<NT, FO, false>, grid, block, 0, st, p, blocks, groups, (int)jobs);
}

// What a call costs one way or another, in us, as measured between 1 x 512 x 8192, 1 x 4096 x 128256, 1 x 28672 x 8192 and
// 4096 x 4096 x 8192.  Of 45 sizes measured on tiles and, few tokens, by rows, to fp32 and bf16, the way that the rule takes is
// the quickest or within 7% of it but for two: 459 x 2171 x 1467 (27.8 us in 5 parts, 24.8 in 2) and 13 x 15616 x 130 (20.0, by rows 16.3).
//
// Rows: every workgroup reads its outputs' weights and its tokens' inputs, at some 6 TB/s from the L2s and behind them, and
// three quarters to a half of that from odd addresses; more workgroups than run at once read the weights at 4.7 TB/s
// (1 x 8192 x 28672: 55 us, 46 on tiles; 1 x 4096 x 128256: 118, 115 on tiles), and a wave waits some 1.6 us for each block of
// a long row (16 x 16384 x 128: 20.7 us, 14.9 on tiles in 16 parts; 8 x 28672 x 1024: 28.1 and 21.5).
//
// Tiles: their blocks' times, which grow with the workgroups that share a compute unit, or the weights' time from memory, and
// some 3.5 us around them; parts take a second kernel, and their way through memory.
struct TileCost {
    int outs, tokens, slots;  // slots: workgroups that a compute unit holds
    float half, one, two;     // us a block with 128 workgroups or fewer, with 256, with 512
};
constexpr TileCost kCosts[] = {{128, 64, 3, 0.74f, 0.86f, 1.32f}, {128, 128, 2, 1.2f, 1.45f, 2.2f}, {256, 128, 1, 1.75f, 2.0f, 0}};
// through registers
constexpr TileCost kCostsStaged[] = {{128, 64, 2, 1.45f, 1.68f, 2.3f}, {128, 128, 2, 2.2f, 2.5f, 3.2f}};
constexpr int kMostParts = 16;
constexpr size_t kMostWorkspace = 64 << 20;

float block_time(const TileCost& c, int64_t jobs) {
    const float at = (float)jobs / 256.0f;
    // (the fullest compute unit counts: 288 workgroups take as long as 512)
    return at <= 0.5f ? c.half : at <= 1 ? c.half + (c.one - c.half) * (2 * at - 1) : c.one + (c.two - c.one) * (float)((jobs - 1) / 256);
}

}  // namespace

// By sizes alone: the workspace is sized before the call's pointers are known, and results of every type are the same sums.
F8Way fc_f8_way(int N, int I, int O) {
    const int blocks = f8_blocks(I);
    F8Way best{};
    float least = 3e38f;
    constexpr int kRows[][2] = {{1, 1}, {1, 2}, {2, 1}, {4, 1}};
    for (const auto& r : kRows) {
        const int64_t jobs = (int64_t)ceil_div(O, 16 * r[1]) * ceil_div(N, 16 * r[0]);
        // 256 of them at once take one's time, and 32 outputs a workgroup are slower where there are fewer
        const float bytes = (float)std::max<int64_t>(jobs, r[1] == 2 ? 256 : 128) * (float)(16 * r[1] + std::min(N, 16 * r[0])) * (float)I;
        const float most = std::max({bytes / 6.3e6f, jobs > 512 ? (float)O * (float)I / 4.7e6f : 0.0f, (float)(blocks / kMostWaves) * 1.6f});
        const float time = 3.0f + most * (I % 4 == 0 ? 1.0f : r[0] == 4 ? 2.1f : 1.3f);
        if (time < least) least = time, best = F8Way{1, r[0], r[1], {}};
    }
    const bool staged = I % kF8Block != 0;
    const float read = (float)O * (float)I / 8e6f;
    for (int c = 0; c < (staged ? 2 : 3); ++c) {
        const TileCost& cost = staged ? kCostsStaged[c] : kCosts[c];
        const int64_t tiles = (int64_t)ceil_div(O, cost.outs) * ceil_div(N, cost.tokens), round = 256 * cost.slots;
        for (int parts = 1; parts <= kMostParts; ++parts) {
            const int run = parts == 1 ? blocks : ceil_div(ceil_div(blocks, parts), 4) * 4;
            const float bytes = (float)parts * N * O * 4.0f;
            if (parts > 1 && (ceil_div(blocks, run) != parts || bytes > (float)kMostWorkspace || tiles * parts > round)) continue;
            const int64_t jobs = tiles * parts, full = jobs / round, rest = jobs % round;
            const float each = (float)full * block_time(cost, round) + (rest ? block_time(cost, rest) : 0.0f);
            const float time = 3.5f + std::max((float)run * each, read) + (parts > 1 ? 3.2f + 0.75e-6f * bytes : 0.0f);
            if (time < least) least = time, best = F8Way{0, 0, 0, F8Tile{cost.outs, cost.tokens, parts, run}};
        }
    }
    return best;
}

size_t fc_f8_workspace(int N, int I, int O) {
    const F8Way way = fc_f8_way(N, I, O);
    return way.rows || way.tile.parts == 1 ? 0 : (size_t)way.tile.parts * N * O * sizeof(float);
}

int launch_fc_f8(const FcF8& p, float* ws, hipStream_t st) {
    if (p.N == 0) return CNN_OK;
    F8Way way = fc_f8_way(p.N, p.I, p.O);
    auto whole = [&](int to) { return (uintptr_t)p.x % to == 0 && (uintptr_t)p.w % to == 0; };
    const bool odd = !whole(4) || p.I % 4 != 0;
    if (!way.rows) {
        const bool vec = whole(16) && p.I % kF8Block == 0;
        if (!vec && way.tile.outs == 256) way.tile.outs = 128;  // whole blocks at addresses that are not
        run_f8_tiles(p, way.tile, vec, ws, st);
    } else if (way.tokens == 1) {
        way.outs == 1 ? run_rows<1, 1>(p, odd, st) : run_rows<1, 2>(p, odd, st);
    } else {
        way.tokens == 2 ? run_rows<2, 1>(p, odd, st) : run_rows<4, 1>(p, odd, st);
    }
    return check_launch("fc_f8");
}

}  // namespace cnn
