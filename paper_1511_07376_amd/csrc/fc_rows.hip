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
// A group of more than 16 RT rows (THIN: 4) takes as many passes over its weights, one after
// another: 256 rows in 64 groups of 2048 x 4096, bf16 on 4 bits, 59 us evenly spread, 144 in one group.
// Bound by HBM where weights are many (16 tokens, 4 of 64 experts of 2048 x 4096, bf16 on 4
// bits: 185 MB in 33.5 to 38 us, 4.9 to 5.5 TB/s), by one chain of load, product and join where
// they are few (one token, 4096 x 4096: 8.9 MB in 4.4 to 4.9 us, of which an empty
// kernel takes 2.3).
#include "fc_operands.h"

#include <algorithm>

namespace cnn {
namespace {

// Thin groups (THIN: up to 4 rows a pass) bring their rows of x to LDS first,
// a wave its own part of the reduction: each value is loaded, and where needed cut
// into parts, by one lane and not by the 16 that use it.
constexpr int kThin = 4;

template <int XT, int WT, int SS>
struct ThinRows {
    static constexpr int ES = kElemBytes<XT>;
    static constexpr int kPlanes = WT == CNN_MX4 ? kParts<XT> : 1;
    static constexpr bool kCut = kPlanes > 1;
    static constexpr int PER = kCut ? 8 : 16 / ES;               // values a vector
    static constexpr int kLoads = kCut && XT == CNN_F32 ? 2 : 1;  // 16-byte loads of one
    static constexpr int kInRow = SS * 128 / PER;                // vectors of a row and step
    static constexpr int kEach = kThin * kInRow / 64;            // of a lane
    static_assert(kThin * kInRow % 64 == 0 && kEach >= 1, "whole vectors a lane");
    static constexpr int kRow = kInRow * 16 + 16;  // bytes in LDS: rows on other banks
    static constexpr int kBytes = kPlanes * kThin * kRow;
};

template <int XT, int WT, int OT, int RT, int SS, bool THIN, bool ODD, bool FULL>
__device__ inline void rows_step(const GroupedFc& p, const char* const* wrow, const uint8_t* const* wscale,
                                 const char* const* xrow, const uint8_t* const* xscale, char* thin, int64_t s, int nb,
                                 f32x4 (&acc)[OT][RT]) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
    constexpr int XLOADS = THIN && ThinRows<XT, WT, SS>::kCut ? 1 : kRunLoads<XT>;
    u32x4 w[OT][SS][kRunLoads<WT>];
    unsigned ws[OT][SS], xs[RT][SS];  // scales, or the last words of runs to be straightened
    u32x4 x[RT][SS][XLOADS];
    // block (32 values) of step t for this lane
    auto block = [&](int t) { return (s * SS + t) * 4 + quad; };
    auto load_mx4 = [&](const char* row, const uint8_t* scale, u32x4* run, unsigned* sc) {
        if constexpr (FULL) {
            unsigned all[SS];
            __builtin_memcpy(all, scale + s * (4 * SS), 4 * SS);
#pragma unroll
            for (int t = 0; t < SS; ++t) {
                run[t] = load16(row + block(t) * 16);
                sc[t] = (all[t] >> (8 * quad)) & 255;
            }
        } else {
#pragma unroll
            for (int t = 0; t < SS; ++t) {
                const bool ok = block(t) < nb;
                run[t] = ok ? load16(row + block(t) * 16) : u32x4{0, 0, 0, 0};
                sc[t] = ok ? scale[block(t)] : 127;
            }
        }
    };
#pragma unroll
    for (int i = 0; i < OT; ++i) {
        if constexpr (WT == CNN_MX4) {
            load_mx4(wrow[i], wscale[i], &w[i][0][0], ws[i]);
        } else {
#pragma unroll
            for (int t = 0; t < SS; ++t) load_run<WT, FULL, ODD>(wrow[i], block(t) * 32, p.I, w[i][t], ws[i][t]);
        }
    }
    using TR = ThinRows<XT, WT, SS>;
    if constexpr (THIN) {
        u32x4 v[TR::kEach][TR::kLoads];
#pragma unroll
        for (int e = 0; e < TR::kEach; ++e) {
            const int64_t k = s * SS * 128 + (e * 64 + lane) % TR::kInRow * TR::PER;
            const char* src = xrow[e] + k * TR::ES;
            if (FULL || k + TR::PER <= p.I) {
#pragma unroll
                for (int h = 0; h < TR::kLoads; ++h) v[e][h] = load16(src + h * 16);
            } else {
                load_edge<XT, TR::kLoads>(src, (int)max(p.I - k, (int64_t)0), k, v[e]);
            }
        }
        // the reads of the step before are done: a wave's LDS accesses run in order
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int e = 0; e < TR::kEach; ++e) {
            char* dst = thin + (e * 64 + lane) / TR::kInRow * TR::kRow + (e * 64 + lane) % TR::kInRow * 16;
            if constexpr (TR::kCut) {
                u32x4 part[TR::kPlanes];
                cut_parts<XT>(v[e], part);
#pragma unroll
                for (int q = 0; q < TR::kPlanes; ++q) *reinterpret_cast<u32x4*>(dst + q * kThin * TR::kRow) = part[q];
            } else {
                *reinterpret_cast<u32x4*>(dst) = v[e][0];
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        if constexpr (!TR::kCut) {
#pragma unroll
            for (int t = 0; t < SS; ++t)
#pragma unroll
                for (int j = 0; j < kRunLoads<XT>; ++j)
                    x[0][t][j] = *reinterpret_cast<const u32x4*>(thin + l16 % kThin * TR::kRow + (t * 128 + quad * 32) * TR::ES + j * 16);
        }
    } else {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            if constexpr (XT == CNN_MX4) {
                load_mx4(xrow[r], xscale[r], &x[r][0][0], xs[r]);
            } else {
#pragma unroll
                for (int t = 0; t < SS; ++t) load_run<XT, FULL, ODD>(xrow[r], block(t) * 32, p.I, x[r][t], xs[r][t]);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < SS; ++t) {
        if constexpr (WT != CNN_MX4) {
#pragma unroll
            for (int i = 0; i < OT; ++i) straighten_run<WT, FULL, ODD>(wrow[i], w[i][t], ws[i][t]);
        }
        if constexpr (XT != CNN_MX4 && !THIN) {
#pragma unroll
            for (int r = 0; r < RT; ++r) straighten_run<XT, FULL, ODD>(xrow[r], x[r][t], xs[r][t]);
        }
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
                    u32x4 part[RT][kParts<XT>];
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        if constexpr (THIN && TR::kCut) {
#pragma unroll
                            for (int q = 0; q < kParts<XT>; ++q)
                                part[r][q] = *reinterpret_cast<const u32x4*>(thin + (q * kThin + l16 % kThin) * TR::kRow + (t * 16 + quad * 4 + j) * 16);
                        } else {
                            cut_parts<XT>(&x[r][t][XT == CNN_F32 ? 2 * j : j], part[r]);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < OT; ++i) {
                        const bf16x8 wv = decode8(w[i][t][0][j], mx4_scale(ws[i][t]));
#pragma unroll
                        for (int r = 0; r < RT; ++r)
#pragma unroll
                            for (int q = kParts<XT> - 1; q >= 0; --q)
                                acc[i][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, __builtin_bit_cast(bf16x8, part[r][q]), acc[i][r], 0, 0, 0);
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

template <int XT, int WT, int OT, int RT, int SS, int NW, bool THIN, bool ODD>
__global__ void __launch_bounds__(64 * NW) fc_rows(GroupedFc p, int units, int cols, FastDiv f_cols) {
    constexpr int ROWS = THIN ? kThin : 16 * RT, OUTS = 16 * OT;
    static_assert(!THIN || (RT == 1 && XT != CNN_MX4), "thin rows are wide");
    using TR = ThinRows<XT, WT, SS>;
    constexpr int XPTRS = THIN ? TR::kEach : RT;
    __shared__ __attribute__((aligned(16))) char thin[THIN ? NW * TR::kBytes : 16];
    __shared__ __attribute__((aligned(16))) float part[NW][OT * RT][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int l16 = lane & 15;
    const int nb = (int)(((int64_t)p.I + 31) / 32);
    const int64_t xbytes = XT == CNN_MX4 ? (int64_t)nb * 16 : (int64_t)p.I * kElemBytes<XT>;
    const int64_t wbytes = WT == CNN_MX4 ? (int64_t)nb * 16 : (int64_t)p.I * kElemBytes<WT>;
    const int64_t span = SS * 128;
    const int64_t full = p.I / span, steps = (p.I + span - 1) / span;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int g = (int)fdiv((unsigned)u, f_cols);
        const int o0 = ((int)u - g * cols) * OUTS;
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
            const char* xrow[XPTRS];
            const uint8_t* xscale[XPTRS];
#pragma unroll
            for (int r = 0; r < XPTRS; ++r) {
                const int row = THIN ? (r * 64 + lane) / TR::kInRow : 16 * r + l16;
                const size_t at = (size_t)max(source_row(p, (int)min(row0 + row, (int64_t)hi - 1)), 0);
                xrow[r] = (const char*)p.x + at * xbytes;
                xscale[r] = p.xs + at * nb;
            }
            f32x4 acc[OT][RT];
#pragma unroll
            for (int i = 0; i < OT; ++i)
#pragma unroll
                for (int r = 0; r < RT; ++r) acc[i][r] = f32x4{0, 0, 0, 0};
            // what the epilogue needs of memory is on its way before the weights are
            constexpr int EACH = (ROWS * OUTS + 64 * NW - 1) / (64 * NW);
            float bias[EACH];
            bool none[EACH];
#pragma unroll
            for (int c = 0; c < EACH; ++c) {
                const int e = threadIdx.x + c * 64 * NW;
                const int64_t m = min(row0 + e / OUTS, (int64_t)hi - 1), o = min((int64_t)o0 + e % OUTS, (int64_t)p.O - 1);
                bias[c] = p.bias ? p.bias[(size_t)g * p.O + o] : 0.0f;
                none[c] = p.rows && source_row(p, (int)m) < 0;
            }
            int64_t s = wave;
            for (; s < full; s += NW) rows_step<XT, WT, OT, RT, SS, THIN, ODD, true>(p, wrow, wscale, xrow, xscale, thin + wave * TR::kBytes * THIN, s, nb, acc);
            if (s < steps) rows_step<XT, WT, OT, RT, SS, THIN, ODD, false>(p, wrow, wscale, xrow, xscale, thin + wave * TR::kBytes * THIN, s, nb, acc);
#pragma unroll
            for (int i = 0; i < OT; ++i)
#pragma unroll
                for (int r = 0; r < RT; ++r) *reinterpret_cast<f32x4*>(&part[wave][i * RT + r][lane * 4]) = acc[i][r];
            __syncthreads();
#pragma unroll
            for (int c = 0; c < EACH; ++c) {
                const int e = threadIdx.x + c * 64 * NW;
                const int row = e / OUTS, o = e % OUTS;
                const int64_t m = row0 + row;
                if (e < ROWS * OUTS && m < hi && (int64_t)o0 + o < p.O) {
                    const int tile = (o / 16) * RT + row / 16;
                    const int at = ((o % 16) / 4 * 16 + row % 16) * 4 + o % 4;
                    float v = 0.0f;
#pragma unroll
                    for (int w = 0; w < NW; ++w) v += part[w][tile][at];
                    v = (none[c] ? 0.0f : v) + bias[c];
                    if (p.relu) v = v > 0.0f ? v : 0.0f;
                    if constexpr (XT == CNN_MX4) store_result(p.y_type, p.y, (size_t)m * p.O + o0 + o, v);
                    else store_result<XT>(p.y, (size_t)m * p.O + o0 + o, v);
                }
            }
            __syncthreads();
        }
    }
}

template <int XT, int WT, int OT, int RT, int SS, int NW, bool THIN>
void start(const GroupedFc& p, hipStream_t st) {
    const int cols = ceil_div(p.O, 16 * OT);
    const int units = p.G * cols;  // below 2^31: checked with the call's arguments
    const dim3 grid((unsigned)std::min(units, 1 << 22)), block(64 * NW);
    constexpr bool kX16 = XT == CNN_BF16 || XT == CNN_F16, kW16 = kX16 && WT != CNN_MX4;
    // rows of 16-bit values at addresses that are no multiples of 4 (thin ones of x: few loads)
    if constexpr (kW16 || (kX16 && !THIN)) {
        if (p.I % 2 || (uintptr_t)p.x % 4 || (kW16 && (uintptr_t)p.w % 4)) {
            enqueue(fc_rows<XT, WT, OT, RT, SS, NW, THIN, true>, grid, block, 0, st, p, units, cols, make_fastdiv(cols));
            return;
        }
    }
    enqueue(fc_rows<XT, WT, OT, RT, SS, NW, THIN, false>, grid, block, 0, st, p, units, cols, make_fastdiv(cols));
}

// The variant of a call.  Wide weights: a workgroup of 8 waves for 16 outputs.
// 4-bit weights: the same where there are few workgroups, with two steps of loads in
// flight a wave (one token, 4096 x 4096: 4.5 us; with 32 outputs a workgroup
// 6.4); from 1024 workgroups on 32 outputs share the rows of x, and a wave
// takes about four steps, so that fewer waves meet in LDS (16 tokens, 4 of 64
// experts of 2048 x 4096, side by side: 38.7 us; 16 outputs and 8 waves 63).  Short reductions leave
// all but the first waves without a step (13 tokens, 6 of 115 experts of 64 x 2752: bf16
// 39.9 us with 8 waves, 12.1 with 2, 8.7 with 1, on 4-bit weights 11.5 with 2, 8.1 with 1; of
// 512 x 1000 18.6, 11.8 and 13.4; 40 tokens, 8 experts of 512 x 1024, fp32 on 4-bit
// weights 7.0, 5.9 and 6.3).
template <int XT, int WT>
void choose(const GroupedFc& p, hipStream_t st) {
    const bool thin = XT != CNN_MX4 && ceil_div64(p.M, p.G) <= kThin;
    // groups without rows cost next to nothing
    const bool many = (int64_t)std::min(p.G, p.M) * ceil_div(p.O, 16) >= 1024;
    if constexpr (WT == CNN_MX4) {
        if constexpr (XT != CNN_MX4) {
            if (thin) {
                if (p.I <= 256) many ? start<XT, WT, 2, 1, 2, 1, true>(p, st) : start<XT, WT, 1, 1, 2, 1, true>(p, st);
                else if (!many) p.I <= 512 ? start<XT, WT, 1, 1, 2, 2, true>(p, st) : start<XT, WT, 1, 1, 2, 8, true>(p, st);
                else if (p.I <= 2048) start<XT, WT, 2, 1, 2, 2, true>(p, st);
                else start<XT, WT, 2, 1, 2, 4, true>(p, st);
                return;
            }
        }
        if constexpr (XT != CNN_F32) {
            if (ceil_div64(p.M, p.G) > 16) {
                if (many) start<XT, WT, 2, 2, 2, 4, false>(p, st);
                else start<XT, WT, 1, 2, 2, 8, false>(p, st);
                return;
            }
        }
        if constexpr (XT == CNN_MX4) {
            // with more rows the epilogue takes 4 waves (58 groups of 16 rows, 145 x 384: 8.4 us against 9.9)
            if (many && p.I <= 512 && ceil_div64(p.M, p.G) <= 8) return start<XT, WT, 2, 1, 2, 2, false>(p, st);
        }
        if (many) start<XT, WT, 2, 1, 2, 4, false>(p, st);
        else if (p.I <= 512) start<XT, WT, 1, 1, 2, 2, false>(p, st);
        else start<XT, WT, 1, 1, 2, 8, false>(p, st);
    } else {
        constexpr int SS = WT == CNN_F32 ? 1 : 2;  // 8 loads of a weight row in flight a lane
        if (p.I <= 128) thin ? start<XT, WT, 1, 1, 1, 1, true>(p, st) : start<XT, WT, 1, 1, SS, 1, false>(p, st);
        else if (p.I <= (WT == CNN_F32 && !many ? 512 : 1024)) thin ? start<XT, WT, 1, 1, 1, 2, true>(p, st) : start<XT, WT, 1, 1, SS, 2, false>(p, st);
        else thin ? start<XT, WT, 1, 1, 1, 8, true>(p, st) : start<XT, WT, 1, 1, SS, 8, false>(p, st);
    }
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
