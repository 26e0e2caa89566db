// Products on groups of many rows: TM x TN tiles, operands staged in LDS.
//
// A workgroup takes TM rows of a group and TN of its outputs and walks the
// reduction in slabs of BK values.  While the matrix cores work on one slab, the
// next one is on its way into the other LDS buffer: rows of whole 16-byte
// vectors are copied there by the load instruction itself, other rows
// (widths or addresses that are not) go through registers, and so do inputs
// that are cut into bfloat16 parts, each value once a workgroup.  Weights of 4
// bits stay 4 bits in LDS and become bfloat16 in the registers of the wave
// that uses them.
//
// LDS rows are 32 to 256 bytes without padding (the copying loads write 64
// consecutive vectors); the 16-byte vectors of a row are exchanged by an XOR with
// some bits of the row, so that lanes on consecutive rows read different banks.
#pragma once

#include "fc_operands.h"

#include <algorithm>

namespace cnn {

struct TileParams {
    GroupedFc fc;
    int cols;          // tiles across the outputs
    int splits;        // parts of the reduction: above 1, sums go to `partial`
    int pairs;         // pairs of slabs a split
    float* partial;    // [splits][M][O]
};

static __device__ const u32x4 kZeroVector = {0, 0, 0, 0};

// The XOR of a row's vectors, C vectors a row.
template <int C>
__device__ constexpr int vector_swap(int row) {
    return C == 16 ? row & 15 : C == 8 ? (row >> 1) & 7 : C == 4 ? (row >> 1) & 3 : (row >> 2) & 1;
}

template <int XT, int WT>
struct Slab {
    static constexpr bool kCut = WT == CNN_MX4 && (XT == CNN_F32 || XT == CNN_F16);
    static constexpr int BK = XT == CNN_MX4 ? 256 : WT == CNN_MX4 ? 64 : XT == CNN_F32 ? 32 : 64;
    static constexpr int kPlanes = kCut ? kParts<XT> : 1;
    static constexpr int AROW = XT == CNN_MX4 ? BK / 2 : kCut ? BK * 2 : BK * kElemBytes<XT>;  // bytes in LDS
    static constexpr int BROW = WT == CNN_MX4 ? BK / 2 : BK * kElemBytes<WT>;
    static constexpr int AC = AROW / 16, BC = BROW / 16;
};

// Number of tiles of TM rows in all groups, and tile t among them.
template <int TM>
struct TileFinder {
    const GroupedFc& p;
    int lane = threadIdx.x & 63;

    __device__ int tiles_of(int base, int& lo, int& end) const {
        lo = end = 0;
        if (base + lane < p.G) group_rows(p.offsets, base + lane, p.M, lo, end);
        return (int)(((unsigned)(end - lo) + TM - 1) / TM);
    }
    __device__ int64_t total() const {
        if (!p.offsets) return ((int64_t)p.M + TM - 1) / TM;
        int64_t sum = 0;
        for (int base = 0; base < p.G; base += 64) {
            int lo, end;
            int t = tiles_of(base, lo, end);
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) t += __shfl_xor(t, off);
            sum += t;
        }
        return sum;
    }
    __device__ void find(int64_t t, int& g, int& row0, int& hi) const {
        g = 0;
        row0 = 0;
        hi = 0;
        if (!p.offsets) {
            row0 = (int)(t * TM);
            hi = p.M;
            return;
        }
        int64_t before = 0;
        for (int base = 0; base < p.G; base += 64) {
            int lo, end;
            const int tiles = tiles_of(base, lo, end);
            int incl = tiles;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const int u = __shfl_up(incl, off);
                if (lane >= off) incl += u;
            }
            const unsigned long long past = __ballot(before + incl > t);
            if (past) {
                const int at = __builtin_ctzll(past);
                const int first = (int)(t - before) - (__shfl(incl, at) - __shfl(tiles, at));
                g = __builtin_amdgcn_readfirstlane(base + at);
                row0 = __builtin_amdgcn_readfirstlane(__shfl(lo, at) + first * TM);
                hi = __builtin_amdgcn_readfirstlane(__shfl(end, at));
                return;
            }
            before += __shfl(incl, 63);
        }
    }
};

// One operand's share of a work-item: the vectors of a slab it fetches.
// DIRECT: copied to LDS by the load.  Otherwise load() brings them to registers and
// store() writes them, as they are or cut into planes.
template <int T, int ROWS, int C, int BK, int NT, bool DIRECT, int PLANES>
struct Fetch {
    static constexpr int kVectors = ROWS * C / NT;  // LDS vectors (of one plane) a work-item
    static_assert(ROWS * C % NT == 0, "whole vectors a work-item");
    static constexpr int PER = T == CNN_MX4 ? 32 : PLANES > 1 ? 8 : 16 / kElemBytes<T>;  // values a vector
    static constexpr int kLoads = PLANES > 1 && T == CNN_F32 ? 2 : 1;                    // 16-byte loads a vector
    const char* ptr[kVectors];  // this work-item's vector of slab 0
    u32x4 reg[DIRECT ? 1 : kVectors * kLoads];

    static __device__ int row_of(int i) { return (i * NT + (int)threadIdx.x) / C; }
    static __device__ int vector_of(int i) {
        return ((i * NT + (int)threadIdx.x) % C) ^ vector_swap<C>(row_of(i));
    }
    static __device__ constexpr int bytes(int values) { return T == CNN_MX4 ? values / 2 : values * kElemBytes<T>; }

    // Slab s; `cols`: values of a row (mx4: of its whole blocks).
    __device__ void load(int64_t s, int cols, char* lds) {
        const bool full = (s + 1) * BK <= cols;
        const int64_t ahead = s * bytes(BK);
        if constexpr (DIRECT) {
#pragma unroll
            for (int i = 0; i < kVectors; ++i) {
                const char* src = ptr[i] + ahead;
                if (!full && s * BK + vector_of(i) * PER >= cols) src = (const char*)&kZeroVector;
                // 64 lanes write 64 consecutive vectors from here on
                char* dst = lds + (i * NT + (int)(threadIdx.x & ~63u)) * 16;
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                                 (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
            }
        } else if (full) {
#pragma unroll
            for (int i = 0; i < kVectors * kLoads; ++i) reg[i] = load16(ptr[i / kLoads] + ahead + i % kLoads * 16);
        } else {
#pragma unroll
            for (int i = 0; i < kVectors; ++i)
                load_edge<T, kLoads>(ptr[i] + ahead, (int)min(cols - s * BK - vector_of(i) * PER, (int64_t)PER), reg + i * kLoads);
        }
    }
    __device__ void store(char* lds) {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int i = 0; i < kVectors; ++i) {
                char* dst = lds + (i * NT + (int)threadIdx.x) * 16;
                if constexpr (PLANES == 1) {
                    *reinterpret_cast<u32x4*>(dst) = reg[i];
                } else {
                    u32x4 part[PLANES];
                    cut_parts<T>(reg + i * kLoads, part);
#pragma unroll
                    for (int q = 0; q < PLANES; ++q) *reinterpret_cast<u32x4*>(dst + q * ROWS * C * 16) = part[q];
                }
            }
        }
    }
};

// The scale bytes of an mx4 operand's fragment rows for two slabs (N bytes).
template <int N>
struct Scales {
    static constexpr int W = N / 4;
    unsigned word[W];
    // blocks [at, at + N) of a row of nb
    __device__ void load(const uint8_t* row, int64_t at, int nb) {
        if (at + N <= nb) {
            if constexpr (N == 16) {
                const u32x4 v = load16(row + at);
#pragma unroll
                for (int i = 0; i < 4; ++i) word[i] = v[i];
            } else {
                __builtin_memcpy(word, row + at, N);
            }
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                unsigned v = 0;
#pragma unroll
                for (int b = 0; b < 4; ++b) v |= (unsigned)(at + 4 * i + b < nb ? row[at + 4 * i + b] : 127) << (8 * b);
                word[i] = v;
            }
        }
    }
};

// All loads of this wave have landed, and all its LDS reads are done; then
// all waves'.
__device__ inline void slab_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// The first `count` of 8 neighbours.
template <typename T>
__device__ inline void store_row8(T* dst, const float* v, int count) {
    if (count >= 8) {
        constexpr int N = 16 / (int)sizeof(T);
#pragma unroll
        for (int h = 0; h < 8 / N; ++h) {
            T part[N];
#pragma unroll
            for (int c = 0; c < N; ++c) part[c] = from_f32<T>(v[h * N + c]);
            u32x4 u;
            __builtin_memcpy(&u, part, 16);
            store16(dst + h * N, u);
        }
    } else {
#pragma unroll
        for (int c = 0; c < 8; ++c)
            if (c < count) dst[c] = from_f32<T>(v[c]);
    }
}

// Two waves a SIMD: 256 registers each.
template <int XT, int WT, int WM, int WN, int FM, int FN, bool VEC>
__global__ void __launch_bounds__(64 * WM * WN, 2) fc_tiles(TileParams tp) {
    using S = Slab<XT, WT>;
    constexpr int TM = WM * FM * 32, TN = WN * FN * 32, NT = 64 * WM * WN, BK = S::BK;
    constexpr bool ADIRECT = XT == CNN_MX4 || (VEC && !S::kCut), BDIRECT = WT == CNN_MX4 || VEC;
    constexpr int APLANE = TM * S::AROW;
    constexpr int NS = 2 * BK / 32;  // scales a row and pair of slabs
    __shared__ __attribute__((aligned(16))) char sA0[APLANE * S::kPlanes], sA1[APLANE * S::kPlanes];
    __shared__ __attribute__((aligned(16))) char sB0[TN * S::BROW], sB1[TN * S::BROW];
    __shared__ int sRow[TM];

    const GroupedFc& p = tp.fc;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm = wave / WN, wn = wave % WN, half = lane >> 5, l32 = lane & 31;

    // Workgroups go to the eight XCDs in turn; each XCD gets a contiguous run
    // of tiles, in bands of 4 rows of tiles walked column by column, so that
    // neighbours share operands in its L2.
    const TileFinder<TM> finder{p};
    const int64_t row_tiles = finder.total();
    const int64_t tiles = row_tiles * tp.cols, jobs = tiles * tp.splits;
    for (int64_t b = blockIdx.x; b < jobs; b += gridDim.x) {
        const int64_t xcd = b % 8, each = jobs / 8, more = jobs % 8;
        const int64_t job = xcd * each + min(xcd, more) + b / 8;
        const int split = (int)(job / tiles);
        const int64_t tile = job % tiles;
        constexpr int BAND = 4;
        const int64_t band = tile / (BAND * tp.cols), in_band = tile % (BAND * tp.cols);
        const int band_rows = (int)min((int64_t)BAND, row_tiles - band * BAND);
        const int o0 = (int)(in_band / band_rows) * TN;
        int g, row0, hi;
        finder.find(band * BAND + in_band % band_rows, g, row0, hi);

        for (int r = tid; r < TM; r += NT) sRow[r] = (int64_t)row0 + r < hi ? source_row(p, row0 + r) : -1;
        __syncthreads();

        const int nb = (int)(((int64_t)p.I + 31) / 32);
        const int acols = XT == CNN_MX4 ? nb * 32 : p.I, bcols = WT == CNN_MX4 ? nb * 32 : p.I;
        const int64_t abytes = XT == CNN_MX4 ? (int64_t)nb * 16 : (int64_t)p.I * kElemBytes<XT>;
        const int64_t bbytes = WT == CNN_MX4 ? (int64_t)nb * 16 : (int64_t)p.I * kElemBytes<WT>;
        using FetchA = Fetch<XT, TM, S::AC, BK, NT, ADIRECT, S::kPlanes>;
        using FetchB = Fetch<WT, TN, S::BC, BK, NT, BDIRECT, 1>;
        FetchA fa;
        FetchB fb;
#pragma unroll
        for (int i = 0; i < FetchA::kVectors; ++i)
            fa.ptr[i] = (const char*)p.x + (int64_t)max(sRow[FetchA::row_of(i)], 0) * abytes + FetchA::bytes(FetchA::vector_of(i) * FetchA::PER);
#pragma unroll
        for (int i = 0; i < FetchB::kVectors; ++i)
            fb.ptr[i] = (const char*)p.w + ((int64_t)g * p.O + min((int64_t)o0 + FetchB::row_of(i), (int64_t)p.O - 1)) * bbytes +
                        FetchB::bytes(FetchB::vector_of(i) * FetchB::PER);
        const uint8_t* as[XT == CNN_MX4 ? FM : 1];
        const uint8_t* bs[WT == CNN_MX4 ? FN : 1];
        if constexpr (XT == CNN_MX4) {
#pragma unroll
            for (int i = 0; i < FM; ++i) as[i] = p.xs + (int64_t)max(sRow[wm * FM * 32 + i * 32 + l32], 0) * nb;
        }
        if constexpr (WT == CNN_MX4) {
#pragma unroll
            for (int j = 0; j < FN; ++j)
                bs[j] = p.ws + ((int64_t)g * p.O + min((int64_t)o0 + wn * FN * 32 + j * 32 + l32, (int64_t)p.O - 1)) * nb;
        }
        Scales<NS> asc[XT == CNN_MX4 ? FM : 1], bsc[WT == CNN_MX4 ? FN : 1];
        auto load_scales = [&](int64_t pair) {
            if constexpr (XT == CNN_MX4) {
#pragma unroll
                for (int i = 0; i < FM; ++i) asc[i].load(as[i], pair * NS, nb);
            }
            if constexpr (WT == CNN_MX4) {
#pragma unroll
                for (int j = 0; j < FN; ++j) bsc[j].load(bs[j], pair * NS, nb);
            }
        };

        f32x16 acc[FM][FN];
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;

        // this lane's first vector of a fragment; those of later steps are an XOR away
        const int arow = (wm * FM * 32 + l32) * S::AROW, brow = (wn * FN * 32 + l32) * S::BROW;
        const int aswap = vector_swap<S::AC>(l32), bswap = vector_swap<S::BC>(l32);
        // scales cur, next: of the pair of slabs at work and of the one after
        auto compute = [&](const char* A, const char* B, int in_pair, const Scales<NS>* xa, const Scales<NS>* wb) {
            auto avec = [&](int plane, int i, int v, int hv) {
                return *reinterpret_cast<const u32x4*>(A + plane * APLANE + i * 32 * S::AROW + arow + (((half * hv) ^ aswap ^ v) * 16));
            };
            auto bvec = [&](int j, int v, int hv) {
                return *reinterpret_cast<const u32x4*>(B + j * 32 * S::BROW + brow + (((half * hv) ^ bswap ^ v) * 16));
            };
            if constexpr (XT == CNN_MX4) {
                // blocks 2 t + half: bytes 0, 2, 4, 6 or 1, 3, 5, 7 of a slab's eight
                const unsigned pick = half ? 0x07050301u : 0x06040200u;
                unsigned sa[FM], sb[FN];
#pragma unroll
                for (int i = 0; i < FM; ++i) sa[i] = __builtin_amdgcn_perm(xa[i].word[2 * in_pair + 1], xa[i].word[2 * in_pair], pick);
#pragma unroll
                for (int j = 0; j < FN; ++j) sb[j] = __builtin_amdgcn_perm(wb[j].word[2 * in_pair + 1], wb[j].word[2 * in_pair], pick);
#define CNN_STEP(t)                                                                                                      \
    {                                                                                                                    \
        u32x4 a[FM], b[FN];                                                                                              \
        _Pragma("unroll") for (int i = 0; i < FM; ++i) a[i] = avec(0, i, 2 * t, 1);                                      \
        _Pragma("unroll") for (int j = 0; j < FN; ++j) b[j] = bvec(j, 2 * t, 1);                                         \
        _Pragma("unroll") for (int i = 0; i < FM; ++i) _Pragma("unroll") for (int j = 0; j < FN; ++j) acc[i][j] =        \
            __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx4_operand(a[i]), mx4_operand(b[j]), acc[i][j], 4, 4, t,    \
                                                            (int)sa[i], t, (int)sb[j]);                                  \
    }
                CNN_STEP(0) CNN_STEP(1) CNN_STEP(2) CNN_STEP(3)
#undef CNN_STEP
            } else if constexpr (WT == CNN_MX4) {
                // two blocks a slab, one for each half of the lanes
                u32x4 raw[FN];
                float sc[FN];
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    raw[j] = bvec(j, 0, 1);
                    sc[j] = mx4_scale((wb[j].word[0] >> (16 * in_pair + 8 * half)) & 255);
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    bf16x8 b[FN];
#pragma unroll
                    for (int j = 0; j < FN; ++j) b[j] = decode8(raw[j][t], sc[j]);
#pragma unroll
                    for (int q = S::kPlanes - 1; q >= 0; --q) {
                        u32x4 a[FM];
#pragma unroll
                        for (int i = 0; i < FM; ++i) a[i] = avec(q, i, t, 4);
#pragma unroll
                        for (int i = 0; i < FM; ++i)
#pragma unroll
                            for (int j = 0; j < FN; ++j)
                                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[i]), b[j], acc[i][j], 0, 0, 0);
                    }
                }
            } else {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    u32x4 a[FM], b[FN];
#pragma unroll
                    for (int i = 0; i < FM; ++i) a[i] = avec(0, i, 2 * t, 1);
#pragma unroll
                    for (int j = 0; j < FN; ++j) b[j] = bvec(j, 2 * t, 1);
                    if constexpr (XT == CNN_F32) {
#pragma unroll
                        for (int c = 0; c < 4; ++c)
#pragma unroll
                            for (int i = 0; i < FM; ++i)
#pragma unroll
                                for (int j = 0; j < FN; ++j)
                                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[i][c]), __uint_as_float(b[j][c]), acc[i][j], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int i = 0; i < FM; ++i)
#pragma unroll
                            for (int j = 0; j < FN; ++j) {
                                if constexpr (XT == CNN_BF16)
                                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[i]), __builtin_bit_cast(bf16x8, b[j]), acc[i][j], 0, 0, 0);
                                else
                                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a[i]), __builtin_bit_cast(f16x8, b[j]), acc[i][j], 0, 0, 0);
                            }
                    }
                }
            }
        };

        const int64_t slabs = ((int64_t)max(acols, bcols) + BK - 1) / BK;
        const int64_t first = (int64_t)split * tp.pairs * 2, last = min(first + (int64_t)tp.pairs * 2, slabs);
        if (first < last) {
            fa.load(first, acols, sA0);
            fb.load(first, bcols, sB0);
            load_scales(first / 2);
            fa.store(sA0);
            fb.store(sB0);
        }
        for (int64_t s = first; s < last; s += 2) {
            Scales<NS> xa[XT == CNN_MX4 ? FM : 1], wb[WT == CNN_MX4 ? FN : 1];
            slab_barrier();
            if constexpr (XT == CNN_MX4) {
#pragma unroll
                for (int i = 0; i < FM; ++i) xa[i] = asc[i];
            }
            if constexpr (WT == CNN_MX4) {
#pragma unroll
                for (int j = 0; j < FN; ++j) wb[j] = bsc[j];
            }
            if (s + 1 < last) {
                fa.load(s + 1, acols, sA1);
                fb.load(s + 1, bcols, sB1);
            }
            if (s + 2 < last) load_scales(s / 2 + 1);
            compute(sA0, sB0, 0, xa, wb);
            if (s + 1 < last) {
                fa.store(sA1);
                fb.store(sB1);
            }
            slab_barrier();
            if (s + 2 < last) {
                fa.load(s + 2, acols, sA0);
                fb.load(s + 2, bcols, sB0);
            }
            if (s + 1 < last) compute(sA1, sB1, 1, xa, wb);
            if (s + 2 < last) {
                fa.store(sA0);
                fb.store(sB0);
            }
        }

        // A lane holds rows 8 (v / 4) + 4 half + v % 4 of column l32 of every 32 x
        // 32 block.  Through LDS, 16 rows of the wave's outputs at a time, it gets
        // 8 neighbours of a row: 128-byte lines leave whole.
        constexpr int SW = FN * 32, VROW = SW / 8, RPI = 64 / VROW;  // strip width, its vectors of 8, rows a round
        static_assert(APLANE * S::kPlanes >= WM * WN * 16 * SW * 4, "the strips fit the first buffer");
        __syncthreads();  // all waves are done with it
        float* strip = reinterpret_cast<float*>(sA0) + wave * 16 * SW;
        const int64_t oc = (int64_t)o0 + wn * SW + lane % VROW * 8;  // this lane's first output
        const int count = (int)min((int64_t)8, p.O - oc);
        float bias[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) bias[c] = tp.splits == 1 && p.bias && c < count ? p.bias[(size_t)g * p.O + oc + c] : 0.0f;
        auto finish = [&](auto put) {
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int j = 0; j < FN; ++j)
#pragma unroll
                        for (int v = 0; v < 8; ++v)
                            strip[(8 * (v / 4) + 4 * half + v % 4) * SW + j * 32 + l32] = acc[i][j][8 * h + v];
                    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                    __builtin_amdgcn_wave_barrier();
                    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
                    for (int it = 0; it < 16 / RPI; ++it) {
                        const int sr = it * RPI + lane / VROW;
                        const int r = wm * FM * 32 + i * 32 + 16 * h + sr;
                        float v[8];
                        *reinterpret_cast<f32x4*>(v) = *reinterpret_cast<const f32x4*>(strip + sr * SW + lane % VROW * 8);
                        *reinterpret_cast<f32x4*>(v + 4) = *reinterpret_cast<const f32x4*>(strip + sr * SW + lane % VROW * 8 + 4);
                        const bool none = sRow[r] < 0;
#pragma unroll
                        for (int c = 0; c < 8; ++c) v[c] = none ? 0.0f : v[c];
                        if ((int64_t)row0 + r < hi && count > 0) put((size_t)(row0 + r) * p.O + oc, v);
                    }
                    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                    __builtin_amdgcn_wave_barrier();
                    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                }
        };
        auto result = [&](float* v) {
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                v[c] += bias[c];
                if (p.relu) v[c] = v[c] > 0.0f ? v[c] : 0.0f;
            }
        };
        if (tp.splits > 1) {
            float* dst = tp.partial + (size_t)split * p.M * p.O;
            finish([&](size_t at, float* v) { store_row8(dst + at, v, count); });
        } else if constexpr (XT == CNN_F32) {
            finish([&](size_t at, float* v) { result(v); store_row8((float*)p.y + at, v, count); });
        } else if constexpr (XT == CNN_BF16) {
            finish([&](size_t at, float* v) { result(v); store_row8((bf16_t*)p.y + at, v, count); });
        } else if constexpr (XT == CNN_F16) {
            finish([&](size_t at, float* v) { result(v); store_row8((f16_t*)p.y + at, v, count); });
        } else {
            finish([&](size_t at, float* v) {
                result(v);
                if (p.y_type == CNN_F32) store_row8((float*)p.y + at, v, count);
                else if (p.y_type == CNN_BF16) store_row8((bf16_t*)p.y + at, v, count);
                else store_row8((f16_t*)p.y + at, v, count);
            });
        }
        __syncthreads();  // sRow is the next tile's
    }
}

// Rows and outputs of a tile.
struct TileSize {
    int rows, outs;
};
// The tile, the splits of the reduction and the slab pairs of each for a call; the same whenever the call's
// sizes and types are, so that the workspace is known before.
struct TilePlan {
    int size;    // index into the tile sizes
    int splits, pairs;
};

template <int XT, int WT, int WM, int WN, int FM, int FN>
void start_tiles(const GroupedFc& p, const TilePlan& plan, bool vec, float* partial, hipStream_t st) {
    constexpr int TM = WM * FM * 32, TN = WN * FN * 32;
    const TileParams tp{p, ceil_div(p.O, TN), plan.splits, plan.pairs, partial};
    // groups end inside a tile: at most one more tile each
    const int64_t jobs = (ceil_div64(p.M, TM) + (p.offsets ? p.G : 0)) * tp.cols * plan.splits;
    const dim3 grid((unsigned)std::min<int64_t>(jobs, 1 << 22)), block(64 * WM * WN);
    if constexpr (XT == CNN_MX4) {
        enqueue(fc_tiles<XT, WT, WM, WN, FM, FN, true>, grid, block, 0, st, tp);
    } else {
        if (vec) enqueue(fc_tiles<XT, WT, WM, WN, FM, FN, true>, grid, block, 0, st, tp);
        else enqueue(fc_tiles<XT, WT, WM, WN, FM, FN, false>, grid, block, 0, st, tp);
    }
}

// By tile size: 0: 64 x 128, 1: 128 x 128, 2: 256 x 256 (128 x 256 for inputs cut into parts, whose planes fill LDS).
template <int XT, int WT>
void run_tiles(const GroupedFc& p, const TilePlan& plan, bool vec, float* partial, hipStream_t st) {
    if (plan.size == 0) start_tiles<XT, WT, 1, 4, 2, 1>(p, plan, vec, partial, st);
    else if (plan.size == 1) start_tiles<XT, WT, 2, 2, 2, 2>(p, plan, vec, partial, st);
    else if constexpr (Slab<XT, WT>::kCut) start_tiles<XT, WT, 2, 4, 2, 2>(p, plan, vec, partial, st);
    else start_tiles<XT, WT, 2, 4, 4, 2>(p, plan, vec, partial, st);
}

void run_tiles_f32(const GroupedFc&, const TilePlan&, bool vec, float* partial, hipStream_t);
void run_tiles_16(const GroupedFc&, const TilePlan&, bool vec, float* partial, hipStream_t);
void run_tiles_mx4(const GroupedFc&, const TilePlan&, bool vec, float* partial, hipStream_t);
void run_tiles_wide_mx4(const GroupedFc&, const TilePlan&, bool vec, float* partial, hipStream_t);
void run_tiles_cut(const GroupedFc&, const TilePlan&, bool vec, float* partial, hipStream_t);

}  // namespace cnn
