// Products on groups of few rows (serving: one token to some tens).
//
// The weights are a stream: each is used by a handful of rows, so what
// counts is that enough loads of them are in flight.  A workgroup takes
// 16 OT outputs of one group, its NW waves share the reduction: a wave loads
// SS * 128 values of each of its weight rows at once, brings them to the
// matrix cores against 16 RT rows of x, which come from the caches, and goes
// on SS * 128 * NW further.  The waves' sums meet in LDS and are added in the
// order of the waves, so results do not change from call to call.  The weights
// are the matrix row, the rows of x the column: with one row of x the
// matrix cores idle to 15/16, which costs nothing while the weights arrive.
// A group of more than 16 RT rows takes as many passes over its weights.
#include "fc_operands.h"

#include <algorithm>

namespace cnn {
namespace {

// 128-value steps a wave loads at once: 4 KiB of weights for each 16 outputs
// (8 for fp32).
template <int WT>
constexpr int kSteps = WT == CNN_MX4 ? 4 : WT == CNN_F32 ? 1 : 1;

template <int XT, int WT, int OT, int RT, bool FULL>
__device__ inline void rows_step(const GroupedFc& p, const char* const* wrow, const uint8_t* const* wscale,
                                 const char* const* xrow, const uint8_t* const* xscale, int64_t s, int nb, int quad,
                                 f32x4 (&acc)[OT][RT]) {
    constexpr int SS = kSteps<WT>;
    u32x4 w[OT][SS][kRunLoads<WT>];
    unsigned ws[OT][SS], xs[RT][SS];
    u32x4 x[RT][SS][kRunLoads<XT>];
    // block (32 values) of step t for this lane
    auto block = [&](int t) { return (s * SS + t) * 4 + quad; };
    auto load_mx4 = [&](const char* row, const uint8_t* scale, u32x4* run, unsigned* sc, int stride) {
        if constexpr (FULL && SS == 4) {
            const u32x4 all = load16(scale + s * 16);
#pragma unroll
            for (int t = 0; t < SS; ++t) {
                run[t * stride] = load16(row + block(t) * 16);
                sc[t] = (all[t] >> (8 * quad)) & 255;
            }
        } else {
#pragma unroll
            for (int t = 0; t < SS; ++t) {
                const bool ok = FULL || block(t) < nb;
                run[t * stride] = ok ? load16(row + block(t) * 16) : u32x4{0, 0, 0, 0};
                sc[t] = ok ? scale[block(t)] : 127;
            }
        }
    };
#pragma unroll
    for (int i = 0; i < OT; ++i) {
        if constexpr (WT == CNN_MX4) {
            load_mx4(wrow[i], wscale[i], &w[i][0][0], ws[i], 1);
        } else {
#pragma unroll
            for (int t = 0; t < SS; ++t) load_run<WT, FULL>(wrow[i], block(t) * 32, p.I, w[i][t]);
        }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if constexpr (XT == CNN_MX4) {
            load_mx4(xrow[r], xscale[r], &x[r][0][0], xs[r], 1);
        } else {
#pragma unroll
            for (int t = 0; t < SS; ++t) load_run<XT, FULL>(xrow[r], block(t) * 32, p.I, x[r][t]);
        }
    }
#pragma unroll
    for (int t = 0; t < SS; ++t) {
        if constexpr (XT == CNN_MX4) {
#pragma unroll
            for (int i = 0; i < OT; ++i)
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    acc[i][r] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        mx4_operand(w[i][t][0]), mx4_operand(x[r][t][0]), acc[i][r], 4, 4, 0, (int)ws[i][t], 0, (int)xs[r][t]);
        } else if constexpr (WT == CNN_F32) {
#pragma unroll
            for (int c = 0; c < 32; ++c)
#pragma unroll
                for (int i = 0; i < OT; ++i)
#pragma unroll
                    for (int r = 0; r < RT; ++r)
                        acc[i][r] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[i][t][c / 4][c % 4]),
                                                                         __uint_as_float(x[r][t][c / 4][c % 4]), acc[i][r], 0, 0, 0);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (WT == CNN_MX4) {
                    bf16x8 part[RT][kParts<XT>];
#pragma unroll
                    for (int r = 0; r < RT; ++r) cut_parts<XT>(x[r][t], j, part[r]);
#pragma unroll
                    for (int i = 0; i < OT; ++i) {
                        const bf16x8 wv = decode8(w[i][t][0][j], mx4_scale(ws[i][t]));
#pragma unroll
                        for (int r = 0; r < RT; ++r)
#pragma unroll
                            for (int q = kParts<XT> - 1; q >= 0; --q)
                                acc[i][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, part[r][q], acc[i][r], 0, 0, 0);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < OT; ++i)
#pragma unroll
                        for (int r = 0; r < RT; ++r) {
                            if constexpr (WT == CNN_BF16)
                                acc[i][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[i][t][j]),
                                                                                    __builtin_bit_cast(bf16x8, x[r][t][j]), acc[i][r], 0, 0, 0);
                            else
                                acc[i][r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, w[i][t][j]),
                                                                                   __builtin_bit_cast(f16x8, x[r][t][j]), acc[i][r], 0, 0, 0);
                        }
                }
            }
        }
    }
}

template <int XT, int WT, int OT, int RT, int NW>
__global__ void __launch_bounds__(64 * NW) fc_rows(GroupedFc p, int64_t units, int cols) {
    constexpr int ROWS = 16 * RT, OUTS = 16 * OT;
    __shared__ __attribute__((aligned(16))) float part[NW][OT * RT][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int l16 = lane & 15, quad = lane >> 4;
    const int nb = (int)(((int64_t)p.I + 31) / 32);
    const int64_t xbytes = XT == CNN_MX4 ? (int64_t)nb * 16 : (int64_t)p.I * kElemBytes<XT>;
    const int64_t wbytes = WT == CNN_MX4 ? (int64_t)nb * 16 : (int64_t)p.I * kElemBytes<WT>;
    const int64_t span = kSteps<WT> * 128;
    const int64_t full = p.I / span, steps = (p.I + span - 1) / span;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int g = (int)(u / cols);
        const int o0 = (int)(u % cols) * OUTS;
        int lo = 0, hi = p.M;
        if (p.offsets) group_rows(p.offsets, g, p.M, lo, hi);
        const char* wrow[OT];
        const uint8_t* wscale[OT];
#pragma unroll
        for (int i = 0; i < OT; ++i) {
            const size_t at = (size_t)g * p.O + (size_t)min((int64_t)o0 + 16 * i + l16, (int64_t)p.O - 1);
            wrow[i] = (const char*)p.w + at * wbytes;
            wscale[i] = p.ws + at * nb;
        }
        for (int64_t row0 = lo; row0 < hi; row0 += ROWS) {
            const char* xrow[RT];
            const uint8_t* xscale[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const size_t at = (size_t)max(source_row(p, (int)min(row0 + 16 * r + l16, (int64_t)hi - 1)), 0);
                xrow[r] = (const char*)p.x + at * xbytes;
                xscale[r] = p.xs + at * nb;
            }
            f32x4 acc[OT][RT];
#pragma unroll
            for (int i = 0; i < OT; ++i)
#pragma unroll
                for (int r = 0; r < RT; ++r) acc[i][r] = f32x4{0, 0, 0, 0};
            int64_t s = wave;
            for (; s < full; s += NW) rows_step<XT, WT, OT, RT, true>(p, wrow, wscale, xrow, xscale, s, nb, quad, acc);
            if (s < steps) rows_step<XT, WT, OT, RT, false>(p, wrow, wscale, xrow, xscale, s, nb, quad, acc);
#pragma unroll
            for (int i = 0; i < OT; ++i)
#pragma unroll
                for (int r = 0; r < RT; ++r) *reinterpret_cast<f32x4*>(&part[wave][i * RT + r][lane * 4]) = acc[i][r];
            __syncthreads();
            for (int e = threadIdx.x; e < ROWS * OUTS; e += 64 * NW) {
                const int row = e / OUTS, o = e % OUTS;
                const int64_t m = row0 + row;
                if (m < hi && (int64_t)o0 + o < p.O) {
                    const int tile = (o / 16) * RT + row / 16;
                    const int at = ((o % 16) / 4 * 16 + row % 16) * 4 + o % 4;
                    float v = 0.0f;
#pragma unroll
                    for (int w = 0; w < NW; ++w) v += part[w][tile][at];
                    if (source_row(p, (int)m) < 0) v = 0.0f;
                    if (p.bias) v += p.bias[(size_t)g * p.O + o0 + o];
                    if (p.relu) v = v > 0.0f ? v : 0.0f;
                    if constexpr (XT == CNN_MX4) store_result(p.y_type, p.y, (size_t)m * p.O + o0 + o, v);
                    else store_result<XT>(p.y, (size_t)m * p.O + o0 + o, v);
                }
            }
            __syncthreads();
        }
    }
}

template <int XT, int WT, int OT, int RT, int NW>
void start(const GroupedFc& p, hipStream_t st) {
    const int cols = ceil_div(p.O, 16 * OT);
    const int64_t units = (int64_t)p.G * cols;
    enqueue(fc_rows<XT, WT, OT, RT, NW>, dim3((unsigned)std::min<int64_t>(units, 1 << 22)), dim3(64 * NW), 0, st, p, units, cols);
}

template <int XT, int WT>
void choose(const GroupedFc& p, hipStream_t st) {
    const int each = (int)ceil_div64(p.M, p.G);
    if (each <= 16) start<XT, WT, 1, 1, 8>(p, st);
    else start<XT, WT, 1, 2, 8>(p, st);
}

}  // namespace

int run_fc_rows(const GroupedFc& p, hipStream_t st) {
    if (p.w_type == CNN_MX4) {
        if (p.x_type == CNN_MX4) choose<CNN_MX4, CNN_MX4>(p, st);
        else if (p.x_type == CNN_F32) choose<CNN_F32, CNN_MX4>(p, st);
        else if (p.x_type == CNN_BF16) choose<CNN_BF16, CNN_MX4>(p, st);
        else choose<CNN_F16, CNN_MX4>(p, st);
    } else if (p.x_type == CNN_F32) choose<CNN_F32, CNN_F32>(p, st);
    else if (p.x_type == CNN_BF16) choose<CNN_BF16, CNN_BF16>(p, st);
    else choose<CNN_F16, CNN_F16>(p, st);
    return check_launch("fc_rows");
}

}  // namespace cnn
