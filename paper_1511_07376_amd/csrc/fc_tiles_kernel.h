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
// Bound, where there is work for all compute units, by the copies into LDS: 8192 x 4096 x
// 4096 in bf16 takes 196 us for its copies alone on 256 x 256 tiles (11 TB/s, from
// the L2s and behind them) and 280 on 128 x 128 (15), the products alone 213 (1290
// TFLOP/s); together 4096 tokens, 2 of 8 experts of 4096 x 4096, take 333 (825 TFLOP/s).
// 4 bits on both sides, 2048 x 9216 x 4096: 59 to 67 us (2.3 to 2.6 PFLOP/s), bound by
// products that the compiler moves behind the barrier, where they cover neither copies nor
// reads (matrix cores busy for 25%; 52 registers spilled).  With few workgroups bound by a
// slab's latency, and in fp32 by the matrix cores (4096 tokens, 2 of 8 of 2048 x 2048: 553
// us, 124 of 154 TFLOP/s).
//
// LDS rows are 128 bytes (4-bit weights beside wide inputs: 32) without padding (the
// copying loads write 64 consecutive vectors); the 16-byte vectors of a row are
// exchanged by an XOR with some bits of the row, so that lanes on consecutive rows read
// different banks.
#pragma once

#include "fc_operands.h"

#include <algorithm>
#include <type_traits>
#include <utility>

namespace cnn {

// The tiles of a call, of which only the last few (fewer than run at once) may
// be split along the reduction: into `parts` runs of `run` slabs, so that the
// tail keeps all compute units busy for part of a tile's time instead of some of
// them for all of it, or for one part more instead of one tile.  (With few tiles the
// tail is all there is.)
struct Tail {
    int full;  // tiles before it
    int tiles, parts, run;
};

// Numbers of tiles fit an int: a tile of a group's rows has one row at least, so there
// are no more than rows times tiles across the outputs, each but the last of
// which stands for 128 outputs or more.
struct TileParams {
    GroupedFc fc;
    int cols;        // tiles across the outputs
    int slabs;       // slabs of the reduction
    int unroll;      // slabs the kernel takes at a time
    int slots;       // workgroups that run at once
    int room;        // parts the workspace holds; 0: no tile is split
    float* partial;  // sums of the tail's parts, a tile each
    float slab_ns;   // what the number of parts is chosen on: a slab's time,
    float share;     // how much of a compute unit's time a workgroup fills,
    float part_ns;   // and the time of a part to be written and joined
    Tail tail;       // without groups: known to the host
};

constexpr int kMaxParts = 16;
constexpr float kJoinNs = 3000;  // the second kernel's own time
// The time of a tail in `parts`, as bits that compare like it, with the parts in the
// lowest 4 (less one).  fc_tiles and fc_join each work it out and have to agree to the
// last bit: every operation is rounded by itself, whatever stands around it where this is
// inlined.
__host__ __device__ inline unsigned tail_key(const TileParams& tp, int tiles, unsigned parts, int& run) {
#pragma clang fp contract(off)
    const unsigned turns = ((unsigned)tp.slabs + tp.unroll - 1) / (unsigned)tp.unroll;
    run = parts == 1 ? tp.slabs : (int)min((turns + parts - 1) / parts * (unsigned)tp.unroll, (unsigned)tp.slabs);
    const unsigned got = ((unsigned)tp.slabs + run - 1) / (unsigned)run;
    const float jobs = (float)tiles * (float)got;
    const float each = (float)(((unsigned)jobs + 255) / 256);  // of a compute unit
    float time = (float)run * tp.slab_ns * fmaxf(1.0f, each * tp.share);
    if (got > 1) time += kJoinNs + jobs * tp.part_ns;
    if (got != parts || (got > 1 && jobs > (float)tp.room)) time = 3e38f;
    return (__builtin_bit_cast(unsigned, time) & ~15u) | (parts - 1);
}
__host__ __device__ inline Tail make_tail(const TileParams& tp, int tiles) {
    Tail t;
    t.full = (int)((unsigned)tiles / (unsigned)tp.slots) * tp.slots;
    t.tiles = tiles - t.full;
    t.parts = 1;
    t.run = tp.slabs;
    if (tp.room == 0 || t.tiles == 0) return t;
#ifdef __HIP_DEVICE_COMPILE__
    // 16 lanes, a number of parts each
    unsigned key = tail_key(tp, t.tiles, (threadIdx.x & 15) + 1, t.run);
    const int run = t.run;
    unsigned best = key;
    best = min(best, (unsigned)__builtin_amdgcn_mov_dpp((int)best, 0x128, 0xf, 0xf, true));  // row_ror 8, 4, 2, 1
    best = min(best, (unsigned)__builtin_amdgcn_mov_dpp((int)best, 0x124, 0xf, 0xf, true));
    best = min(best, (unsigned)__builtin_amdgcn_mov_dpp((int)best, 0x122, 0xf, 0xf, true));
    best = min(best, (unsigned)__builtin_amdgcn_mov_dpp((int)best, 0x121, 0xf, 0xf, true));
    best = (unsigned)__builtin_amdgcn_readfirstlane((int)best);
    t.parts = (int)(best & 15) + 1;
    t.run = __builtin_amdgcn_readlane(run, t.parts - 1);
#else
    unsigned best = ~0u;
    for (unsigned parts = 1; parts <= kMaxParts; ++parts) {
        int run;
        const unsigned key = tail_key(tp, t.tiles, parts, run);
        if (key < best) best = key, t.parts = (int)parts, t.run = run;
    }
#endif
    return t;
}

static __device__ const u32x4 kZeroVector = {0, 0, 0, 0};

// The XOR of a row's vectors, C vectors a row.
template <int C>
__device__ constexpr int vector_swap(int row) {
    static_assert(C == 8 || C == 2, "rows of 128 bytes, or of 4-bit weights beside wide inputs");
    return C == 8 ? (row >> 1) & 7 : (row >> 2) & 1;
}

// The slabs of a kernel.  VEC: rows of wide operands are whole 16-byte vectors.
// Operands that are copied to LDS by the loads have ST buffers there, so that
// ST - 1 slabs are on their way while one is at work; those that go through
// registers have two, and R slabs on their way in registers.
template <int XT, int WT, int WM, int WN, int FM, int FN, bool VEC>
struct Slab {
    static constexpr bool kCut = WT == CNN_MX4 && (XT == CNN_F32 || XT == CNN_F16);
    static constexpr bool kDecode = WT == CNN_MX4 && XT != CNN_MX4;
    static constexpr bool ADIRECT = XT == CNN_MX4 || (VEC && !kCut), BDIRECT = WT == CNN_MX4 || VEC;
    static constexpr int TM = WM * FM * 32, TN = WN * FN * 32, NT = 64 * WM * WN;
    // steps of a plane's products in a slab (16 values of the 16-bit types, 8 of fp32, 64 of mx4)
    static constexpr int T = 4;
    static constexpr int BK = T * (XT == CNN_MX4 ? 64 : WT == CNN_F32 ? 8 : 16);
    static constexpr int kPlanes = kCut ? kParts<XT> : 1;
    static constexpr int AROW = XT == CNN_MX4 ? BK / 2 : kCut ? BK * 2 : BK * kElemBytes<XT>;  // bytes in LDS
    static constexpr int BROW = WT == CNN_MX4 ? BK / 2 : BK * kElemBytes<WT>;
    static constexpr int AC = AROW / 16, BC = BROW / 16;
    static constexpr int APLANE = TM * AROW;
    // 4 buffers where they fit with another workgroup's beside them (4 waves) or alone (8)
    static constexpr int kRoom = WM * WN > 4 ? 160 * 1024 - 2048 : 80 * 1024 - 1024;
    static constexpr int ST = ((ADIRECT ? 4 : 2) * APLANE * kPlanes + (BDIRECT ? 4 : 2) * TN * BROW) <= kRoom ? 4 : 2;
    static constexpr int AST = ADIRECT ? ST : 2, BST = BDIRECT ? ST : 2;
    static constexpr int R = WM * FM * WN * FN > 16 ? 1 : 2;
    static_assert(R <= ST, "what is awaited is older than what may be on its way");
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
    __device__ int total() const {
        if (!p.offsets) return (int)(((unsigned)p.M + TM - 1) / TM);
        int sum = 0;
        for (int base = 0; base < p.G; base += 64) {
            int lo, end;
            int t = tiles_of(base, lo, end);
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) t += __shfl_xor(t, off);
            sum += t;
        }
        return __builtin_amdgcn_readfirstlane(sum);  // so that what depends on it stays scalar
    }
    __device__ void find(int t, int& g, int& row0, int& hi) const {
        g = 0;
        row0 = 0;
        hi = 0;
        if (!p.offsets) {
            row0 = t * TM;
            hi = p.M;
            return;
        }
        int before = 0;
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
                const int first = t - before - (__shfl(incl, at) - __shfl(tiles, at));
                g = __builtin_amdgcn_readfirstlane(base + at);
                // offsets that are not in order can make more tiles than an int counts
                if ((unsigned)first < (unsigned)__shfl(tiles, at)) {
                    row0 = __builtin_amdgcn_readfirstlane(__shfl(lo, at) + first * TM);
                    hi = __builtin_amdgcn_readfirstlane(__shfl(end, at));
                }
                return;
            }
            before += __builtin_amdgcn_readlane(incl, 63);
        }
    }
};

// Where tile t is: tiles are numbered in bands of 4 rows of tiles, walked column by
// column, so that neighbours share operands in an XCD's L2.
template <int TM, int TN>
__device__ inline void locate_tile(const TileFinder<TM>& finder, int t, int row_tiles, int cols, int& g, int& row0, int& hi, int& o0) {
    constexpr unsigned BAND = 4;
    const unsigned band = (unsigned)t / (BAND * (unsigned)cols), in_band = (unsigned)t % (BAND * (unsigned)cols);
    const unsigned band_rows = min(BAND, (unsigned)row_tiles - band * BAND);
    o0 = (int)(in_band / band_rows) * TN;
    finder.find((int)(band * BAND + in_band % band_rows), g, row0, hi);
}

// One operand's share of a work-item: the vectors of a slab it fetches.
// DIRECT: copied to LDS by the load.  Otherwise load() brings them to registers and
// store() writes them, as they are or cut into planes.
template <int T, int ROWS, int C, int BK, int NT, bool DIRECT, int PLANES, int R>
struct Fetch {
    static constexpr int kVectors = ROWS * C / NT;  // LDS vectors (of one plane) a work-item
    static_assert(ROWS * C % NT == 0, "whole vectors a work-item");
    static constexpr int PER = T == CNN_MX4 ? 32 : PLANES > 1 ? 8 : 16 / kElemBytes<T>;  // values a vector
    static constexpr int kLoads = PLANES > 1 && T == CNN_F32 ? 2 : 1;                    // 16-byte loads a vector
    const char* ptr[kVectors];  // this work-item's vectors of the next slab
    static constexpr int kInstructions = kVectors * kLoads;  // memory instructions a slab
    u32x4 reg[DIRECT ? 1 : R][DIRECT ? 1 : kVectors * kLoads];

    static __device__ int row_of(int i) { return (i * NT + (int)threadIdx.x) / C; }
    static __device__ int vector_of(int i) {
        return ((i * NT + (int)threadIdx.x) % C) ^ vector_swap<C>(row_of(i));
    }
    static __device__ constexpr int bytes(int values) { return T == CNN_MX4 ? values / 2 : values * kElemBytes<T>; }

    // The next slab, s, of rows of `cols` values (mx4: of whole blocks), to LDS or to
    // registers r.
    __device__ void load(int64_t cols, int64_t s, char* lds, int r) {
        const int64_t left = cols - s * BK;
        if (left >= BK) {
#pragma unroll
            for (int i = 0; i < kVectors; ++i) {
                if constexpr (DIRECT) {
                    copy(i, ptr[i], lds);
                } else {
#pragma unroll
                    for (int h = 0; h < kLoads; ++h) reg[r][i * kLoads + h] = load16(ptr[i] + h * 16);
                }
                ptr[i] += bytes(BK);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kVectors; ++i) {
                const int k = vector_of(i) * PER;
                if constexpr (DIRECT) copy(i, k < left ? ptr[i] : (const char*)&kZeroVector, lds);
                else load_edge<T, kLoads>(ptr[i], (int)min(left - k, (int64_t)PER), s * BK + k, reg[r] + i * kLoads);
            }
        }
    }
    // 64 lanes write 64 consecutive vectors
    static __device__ void copy(int i, const char* src, char* lds) {
        char* dst = lds + (i * NT + (int)(threadIdx.x & ~63u)) * 16;
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                         (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
    }
    __device__ void store(char* lds, int r) {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int i = 0; i < kVectors; ++i) {
                char* dst = lds + (i * NT + (int)threadIdx.x) * 16;
                if constexpr (PLANES == 1) {
                    *reinterpret_cast<u32x4*>(dst) = reg[r][i];
                } else {
                    u32x4 part[PLANES];
                    cut_parts<T>(reg[r] + i * kLoads, part);
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
    // blocks [at, at + N) of the row of nb that begins at base + row
    __device__ void load(const uint8_t* base, int row, int at, int nb) {
        const uint8_t* src = base + (unsigned)(row + at);
        if (at + N <= nb) {
            __builtin_memcpy(word, src, N);
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                unsigned v = 0x7f7f7f7fu;  // beside zeros: anything but NaN
#pragma unroll 1
                for (int b = 0; b < 4 && at + 4 * i + b < nb; ++b) v = (v & ~(255u << (8 * b))) | (unsigned)src[4 * i + b] << (8 * b);
                word[i] = v;
            }
        }
    }
};

template <int N>
using Step = std::integral_constant<int, N>;
template <typename F, int... U>
__device__ inline void unroll_steps(F&& f, std::integer_sequence<int, U...>) {
    (f(Step<U>{}), ...);
}
template <int N, typename F>
__device__ inline void unroll_steps(F&& f) {
    unroll_steps(f, std::make_integer_sequence<int, N>{});
}

// All but the wave's last N loads have landed, and all its LDS accesses are
// done; then all waves'.
template <int N>
__device__ inline void slab_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x70);  // vmcnt(N) lgkmcnt(0)
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
    using S = Slab<XT, WT, WM, WN, FM, FN, VEC>;
    constexpr int TM = S::TM, TN = S::TN, NT = S::NT, BK = S::BK, APLANE = S::APLANE, ST = S::ST, R = S::R;
    constexpr int kUnroll = ST;             // slabs: every buffer at a fixed place in the code
    constexpr int NS = kUnroll * BK / 32;   // scales of a row in them
    constexpr int ABYTES = APLANE * S::kPlanes, BBYTES = TN * S::BROW;
    // arrays of their own: the compiler sees that a copy into one does not concern reads of another
    __shared__ __attribute__((aligned(16))) char sA0[ABYTES], sA1[ABYTES], sA2[S::AST > 2 ? ABYTES : 16], sA3[S::AST > 2 ? ABYTES : 16];
    __shared__ __attribute__((aligned(16))) char sB0[BBYTES], sB1[BBYTES], sB2[S::BST > 2 ? BBYTES : 16], sB3[S::BST > 2 ? BBYTES : 16];
    __shared__ int sRow[TM];
    auto abuf = [&](auto slab) -> char* {
        constexpr int i = decltype(slab)::value % S::AST;
        if constexpr (i == 0) return sA0;
        else if constexpr (i == 1) return sA1;
        else if constexpr (i == 2) return sA2;
        else return sA3;
    };
    auto bbuf = [&](auto slab) -> char* {
        constexpr int i = decltype(slab)::value % S::BST;
        if constexpr (i == 0) return sB0;
        else if constexpr (i == 1) return sB1;
        else if constexpr (i == 2) return sB2;
        else return sB3;
    };

    const GroupedFc& p = tp.fc;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm = wave / WN, wn = wave % WN, half = lane >> 5, l32 = lane & 31;

    // Workgroups go to the eight XCDs in turn; each XCD gets a contiguous run of
    // the tiles.
    const TileFinder<TM> finder{p};
    const int row_tiles = finder.total();
    const Tail tail = p.offsets ? make_tail(tp, row_tiles * tp.cols) : tp.tail;
    const int jobs = tail.full + tail.tiles * tail.parts;
    for (int turn = blockIdx.x; turn < jobs; turn += gridDim.x) {
        int tile, part = 0;
        if (turn < tail.full) {
            const int xcd = turn % 8, each = tail.full / 8, more = tail.full % 8;
            tile = xcd * each + min(xcd, more) + turn / 8;
        } else {
            tile = tail.full + (turn - tail.full) % tail.tiles;
            part = (turn - tail.full) / tail.tiles;
        }
        const bool split = turn >= tail.full && tail.parts > 1;
        int g, row0, hi, o0;
        locate_tile<TM, TN>(finder, tile, row_tiles, tp.cols, g, row0, hi, o0);

        for (int r = tid; r < TM; r += NT) sRow[r] = (int64_t)row0 + r < hi ? source_row(p, row0 + r) : -1;
        __syncthreads();

        const int nb = (int)(((int64_t)p.I + 31) / 32);
        const int64_t acols = XT == CNN_MX4 ? (int64_t)nb * 32 : p.I, bcols = WT == CNN_MX4 ? (int64_t)nb * 32 : p.I;
        const int64_t abytes = XT == CNN_MX4 ? (int64_t)nb * 16 : (int64_t)p.I * kElemBytes<XT>;
        const int64_t bbytes = WT == CNN_MX4 ? (int64_t)nb * 16 : (int64_t)p.I * kElemBytes<WT>;
        const int64_t first = split ? (int64_t)part * tail.run : 0, last = split ? min(first + tail.run, (int64_t)tp.slabs) : tp.slabs;
        using FetchA = Fetch<XT, TM, S::AC, BK, NT, S::ADIRECT, S::kPlanes, R>;
        using FetchB = Fetch<WT, TN, S::BC, BK, NT, S::BDIRECT, 1, R>;
        FetchA fa;
        FetchB fb;
#pragma unroll
        for (int i = 0; i < FetchA::kVectors; ++i)
            fa.ptr[i] = (const char*)p.x + (int64_t)max(sRow[FetchA::row_of(i)], 0) * abytes + FetchA::bytes(FetchA::vector_of(i) * FetchA::PER) + first * FetchA::bytes(BK);
#pragma unroll
        for (int i = 0; i < FetchB::kVectors; ++i)
            fb.ptr[i] = (const char*)p.w + ((int64_t)g * p.O + min((int64_t)o0 + FetchB::row_of(i), (int64_t)p.O - 1)) * bbytes +
                        FetchB::bytes(FetchB::vector_of(i) * FetchB::PER) + first * FetchB::bytes(BK);
        // scale rows: offsets from the group's (fewer than 2^31 values, so fewer scales)
        const uint8_t* wscale = p.ws + (int64_t)g * p.O * nb;
        int as[XT == CNN_MX4 ? FM : 1], bs[WT == CNN_MX4 ? FN : 1];
        if constexpr (XT == CNN_MX4) {
#pragma unroll
            for (int i = 0; i < FM; ++i) as[i] = max(sRow[wm * FM * 32 + i * 32 + l32], 0) * nb;
        }
        if constexpr (WT == CNN_MX4) {
#pragma unroll
            for (int j = 0; j < FN; ++j) bs[j] = (int)min((int64_t)o0 + wn * FN * 32 + j * 32 + l32, (int64_t)p.O - 1) * nb;
        }
        // scales of kUnroll slabs: those at work, and those that follow
        Scales<NS> acur[XT == CNN_MX4 ? FM : 1], anext[XT == CNN_MX4 ? FM : 1], bcur[WT == CNN_MX4 ? FN : 1], bnext[WT == CNN_MX4 ? FN : 1];
        auto load_scales = [&](int64_t slab) {
            const int at = (int)(slab * (BK / 32));
            if constexpr (XT == CNN_MX4) {
#pragma unroll
                for (int i = 0; i < FM; ++i) anext[i].load(p.xs, as[i], at, nb);
            }
            if constexpr (WT == CNN_MX4) {
#pragma unroll
                for (int j = 0; j < FN; ++j) bnext[j].load(wscale, bs[j], at, nb);
            }
        };

        f32x16 acc[FM][FN];
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;

        // A slab is U steps: T parts of its reduction, and for cut inputs each of
        // their planes, least first.  A step's fragments are read while the one before
        // is at work.
        constexpr int U = S::T * S::kPlanes;
        // this lane's first vector of a fragment; those of other steps are an XOR away
        const int afirst = (wm * FM * 32 + l32) * S::AROW + ((half * (S::kDecode ? 4 : 1)) ^ vector_swap<S::AC>(l32)) * 16;
        const int bfirst = (wn * FN * 32 + l32) * S::BROW + (half ^ vector_swap<S::BC>(l32)) * 16;
        static_assert(U % 2 == 0, "a step's set is the same in every slab");
        u32x4 a[2][FM], b[2][FN];  // b: of a step, or of a slab (4-bit weights to be decoded)
        bf16x8 wide[S::kDecode ? FN : 1];
        auto read = [&](auto slab, auto step) {
            constexpr int u = decltype(step)::value, t = u / S::kPlanes, q = S::kPlanes - 1 - u % S::kPlanes;
            constexpr int av = (S::kDecode ? t : 2 * t) * 16, bv = S::kDecode ? 0 : 2 * t * 16;
            const char *A = abuf(slab), *B = bbuf(slab);
            int af = afirst, bf = bfirst;
            asm volatile("" : "+v"(af), "+v"(bf));  // one XOR here, not an address for every step in a register
#pragma unroll
            for (int i = 0; i < FM; ++i) a[u % 2][i] = *reinterpret_cast<const u32x4*>(A + q * APLANE + i * 32 * S::AROW + (af ^ av));
            if constexpr (!S::kDecode || u == 0) {
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    b[S::kDecode ? decltype(slab)::value % 2 : u % 2][j] = *reinterpret_cast<const u32x4*>(B + j * 32 * S::BROW + (bf ^ bv));
            }
        };
        auto multiply = [&](auto slab, auto step) {
            constexpr int h = decltype(slab)::value, u = decltype(step)::value, t = u / S::kPlanes, set = u % 2;
            if constexpr (S::kDecode && u % S::kPlanes == 0) {
                // a slab is two blocks, one for each half of the lanes
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    wide[j] = decode8(b[h % 2][j][t], mx4_scale((bcur[j].word[h / 2] >> (16 * (h % 2) + 8 * half)) & 255));
            }
            // mx4: a lane's blocks are 2 t + half: bytes 0 and 2 of two words, shifted by the half
            auto scale = [&](const Scales<NS>& sc) { return (int)(sc.word[(2 * h + t / 2) % Scales<NS>::W] >> (8 * half)); };
            constexpr int REPEAT = XT == CNN_F32 && WT == CNN_F32 ? 4 : 1;
#pragma unroll
            for (int c = 0; c < REPEAT; ++c)
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j) {
                        if constexpr (XT == CNN_MX4)
                            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx4_operand(a[set][i]), mx4_operand(b[set][j]), acc[i][j], 4, 4,
                                                                                        t % 2 * 2, scale(acur[i]), t % 2 * 2, scale(bcur[j]));
                        else if constexpr (S::kDecode)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[set][i]), wide[j], acc[i][j], 0, 0, 0);
                        else if constexpr (XT == CNN_F32)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[set][i][c]), __uint_as_float(b[set][j][c]), acc[i][j], 0, 0, 0);
                        else if constexpr (XT == CNN_BF16)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[set][i]), __builtin_bit_cast(bf16x8, b[set][j]), acc[i][j], 0, 0, 0);
                        else
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a[set][i]), __builtin_bit_cast(f16x8, b[set][j]), acc[i][j], 0, 0, 0);
                    }
            __builtin_amdgcn_sched_barrier(0);
        };
        // Asks for slab s (place `slab` in the unrolled code) of the operands that
        // are copied, or of those that go through registers.
        auto ask_direct = [&](int64_t s, auto slab) {
            if (s >= last) return;
            if constexpr (S::ADIRECT) fa.load(acols, s, abuf(slab), 0);
            if constexpr (S::BDIRECT) fb.load(bcols, s, bbuf(slab), 0);
        };
        auto ask_staged = [&](int64_t s, auto slab) {
            if (s >= last) return;
            if constexpr (!S::ADIRECT) fa.load(acols, s, nullptr, decltype(slab)::value % R);
            if constexpr (!S::BDIRECT) fb.load(bcols, s, nullptr, decltype(slab)::value % R);
        };
        auto put_staged = [&](auto slab) {
            fa.store(abuf(slab), decltype(slab)::value % R);
            fb.store(bbuf(slab), decltype(slab)::value % R);
        };
        // loads that may be on their way when a slab is taken: of ST - 2 later slabs and of R - 1
        constexpr int kDirect = S::ADIRECT * FetchA::kInstructions + S::BDIRECT * FetchB::kInstructions;
        constexpr int kStaged = !S::ADIRECT * FetchA::kInstructions + !S::BDIRECT * FetchB::kInstructions;
        constexpr int kAhead = (ST - 2) * kDirect + (R - 1) * kStaged;
        static_assert(kAhead < 64, "what a wait can count");
        // Slab s, its first step already read.  Before its last step the next slab is made
        // ready, later ones are asked for (this one's buffer is free: all waves have
        // read what they need), and the next one's first step is read: the last step's
        // products cover that.  (Three steps ahead instead of one: no faster.)  follows: there
        // is a next slab.
        auto work = [&](int64_t s, auto slab, auto follows) {
            constexpr int h = decltype(slab)::value;
            unroll_steps<U - 1>([&](auto step) {
                read(slab, Step<decltype(step)::value + 1>{});
                multiply(slab, step);
            });
            if (decltype(follows)::value || s + 1 < last) {
                put_staged(Step<h + 1>{});
                // near the end loads may be fewer than counted on
                if (kAhead > 0 && s + ST + 1 < last) slab_barrier<kAhead>();
                else slab_barrier<0>();
                ask_direct(s + ST, Step<h + ST>{});
                ask_staged(s + 1 + R, Step<h + 1 + R>{});
                if (h == kUnroll - 2 && s + 2 < last) load_scales(s + 2);
                read(Step<(h + 1) % kUnroll>{}, Step<0>{});
            }
            multiply(slab, Step<U - 1>{});
        };
        auto next_scales = [&] {
            if constexpr (XT == CNN_MX4) {
#pragma unroll
                for (int i = 0; i < FM; ++i) acur[i] = anext[i];
            }
            if constexpr (WT == CNN_MX4) {
#pragma unroll
                for (int j = 0; j < FN; ++j) bcur[j] = bnext[j];
            }
        };
        if (first < last) {
            unroll_steps<ST>([&](auto slab) { ask_direct(first + decltype(slab)::value, slab); });
            unroll_steps<R>([&](auto slab) { ask_staged(first + decltype(slab)::value, slab); });
            load_scales(first);
            put_staged(Step<0>{});
            slab_barrier<0>();
            ask_staged(first + R, Step<R>{});
            read(Step<0>{}, Step<0>{});
            // A loop of slabs that are all followed by another one, then the last ones: 2 to 8%
            // faster than one loop that tests for each.
            int64_t s = first;
            for (; s + kUnroll < last; s += kUnroll) {
                next_scales();
                unroll_steps<kUnroll>([&](auto slab) { work(s + decltype(slab)::value, slab, std::true_type{}); });
            }
            next_scales();
            unroll_steps<kUnroll>([&](auto slab) {
                if (s + decltype(slab)::value < last) work(s + decltype(slab)::value, slab, std::false_type{});
            });
        }

        // A lane holds rows 8 (v / 4) + 4 half + v % 4 of column l32 of every 32 x
        // 32 block.  Through LDS, 16 rows of the wave's outputs at a time, it gets
        // 8 neighbours of a row: 128-byte lines leave whole.
        constexpr int SW = FN * 32, VROW = SW / 8, RPI = 64 / VROW;  // strip width, its vectors of 8, rows a round
        constexpr int STRIP = 16 * SW * 4, PER = ABYTES / STRIP;  // strips a buffer
        static_assert(PER > 0 && 2 * PER >= WM * WN, "the strips fit two buffers");
        __syncthreads();  // all waves are done with them
        float* strip = reinterpret_cast<float*>((wave < PER ? sA0 : sA1) + wave % PER * STRIP);
        const int64_t oc = (int64_t)o0 + wn * SW + lane % VROW * 8;  // this lane's first output
        const int count = (int)min((int64_t)8, p.O - oc);
        float bias[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) bias[c] = !split && p.bias && c < count ? p.bias[(size_t)g * p.O + oc + c] : 0.0f;
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
                        if ((int64_t)row0 + r < hi && count > 0) put((size_t)((int64_t)row0 + r) * p.O + oc, r, v);
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
        if (split) {
            float* dst = tp.partial + (int64_t)(turn - tail.full) * (TM * TN) - o0;
            finish([&](size_t, int r, float* v) { store_row8(dst + r * TN + oc, v, 8); });
        } else if constexpr (XT == CNN_F32) {
            finish([&](size_t at, int, float* v) { result(v); store_row8((float*)p.y + at, v, count); });
        } else if constexpr (XT == CNN_BF16) {
            finish([&](size_t at, int, float* v) { result(v); store_row8((bf16_t*)p.y + at, v, count); });
        } else if constexpr (XT == CNN_F16) {
            finish([&](size_t at, int, float* v) { result(v); store_row8((f16_t*)p.y + at, v, count); });
        } else {
            finish([&](size_t at, int, float* v) {
                result(v);
                if (p.y_type == CNN_F32) store_row8((float*)p.y + at, v, count);
                else if (p.y_type == CNN_BF16) store_row8((bf16_t*)p.y + at, v, count);
                else store_row8((f16_t*)p.y + at, v, count);
            });
        }
        __syncthreads();  // sRow is the next tile's
    }
}

// Adds the parts of the tail's tiles, in their order, then bias and ReLU.  A
// work-item takes 4 neighbours, a workgroup 1024 outputs of a tile.
template <int TM, int TN, int YT>
__global__ void __launch_bounds__(256) fc_join(TileParams tp) {
    constexpr int CHUNKS = TM * TN / 1024;
    const GroupedFc& p = tp.fc;
    const TileFinder<TM> finder{p};
    const int row_tiles = finder.total();
    const Tail tail = p.offsets ? make_tail(tp, row_tiles * tp.cols) : tp.tail;
    if (tail.parts < 2) return;
    for (int u = blockIdx.x; u < tail.tiles * CHUNKS; u += gridDim.x) {
        const int t = u / CHUNKS, e = u % CHUNKS * 1024 + (int)threadIdx.x * 4, r = e / TN, c = e % TN;
        int g, row0, hi, o0;
        locate_tile<TM, TN>(finder, tail.full + t, row_tiles, tp.cols, g, row0, hi, o0);
        const int64_t o = (int64_t)o0 + c, m = (int64_t)row0 + r;
        const int count = (int)min((int64_t)4, p.O - o);
        if (m >= hi || count <= 0) continue;
        float bias[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) bias[i] = p.bias && i < count ? p.bias[(size_t)g * p.O + o + i] : 0.0f;
        const float* src = tp.partial + (int64_t)t * (TM * TN) + e;
        f32x4 sum = {0, 0, 0, 0};
#pragma unroll 4
        for (int q = 0; q < tail.parts; ++q) sum += *reinterpret_cast<const f32x4*>(src + (int64_t)q * tail.tiles * (TM * TN));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float v = sum[i] + bias[i];
            if (p.relu) v = v > 0.0f ? v : 0.0f;
            if (i < count) store_result<YT>(p.y, (size_t)m * p.O + o + i, v);
        }
    }
}

// A call's tile size: 32 x 128, 64 x 128, 128 x 128 or 256 x 256; 32 x 128 or 128 x 256
// for inputs cut into parts.
struct TileSize {
    int rows, outs;
    int slots;                      // workgroups that run at once on 256 compute units
    int room;                       // parts of split tiles
    float slab_ns, share, part_ns;  // as TileParams
};

// Wide inputs have results of their own type, 4-bit ones of any.
template <int XT, int TM, int TN>
void start_join(const TileParams& tp, int64_t tiles, hipStream_t st) {
    if (!tp.fc.offsets) tiles = tp.tail.tiles;
    // no more than are there at once (8 a compute unit): the tail of groups can be far shorter than it might (4096
    // tokens, 2 of 8 experts of 2048 x 2048, bf16: 120 us against 129)
    const dim3 grid((unsigned)std::min<int64_t>(std::min<int64_t>(tiles, tp.slots) * (TM * TN / 1024), 2048)), block(256);
    if constexpr (XT != CNN_MX4) enqueue(fc_join<TM, TN, XT>, grid, block, 0, st, tp);
    else if (tp.fc.y_type == CNN_F32) enqueue(fc_join<TM, TN, CNN_F32>, grid, block, 0, st, tp);
    else if (tp.fc.y_type == CNN_BF16) enqueue(fc_join<TM, TN, CNN_BF16>, grid, block, 0, st, tp);
    else enqueue(fc_join<TM, TN, CNN_F16>, grid, block, 0, st, tp);
}

template <int XT, int WT, int WM, int WN, int FM, int FN, bool VEC>
void start_tiles(const GroupedFc& p, const TileSize& size, float* partial, hipStream_t st) {
    using S = Slab<XT, WT, WM, WN, FM, FN, VEC>;
    const int64_t values = XT == CNN_MX4 ? ((int64_t)p.I + 31) / 32 * 32 : p.I;
    TileParams tp{p, ceil_div(p.O, S::TN), (int)ceil_div64(values, S::BK), S::ST, size.slots, size.room, partial, size.slab_ns, size.share, size.part_ns, {}};
    // groups end inside a tile: at most one more tile each
    const int64_t tiles = (ceil_div64(p.M, S::TM) + (p.offsets ? p.G : 0)) * tp.cols;
    if (!p.offsets) tp.tail = make_tail(tp, (int)tiles);
    const int64_t jobs = p.offsets ? tiles + size.room : tp.tail.full + (int64_t)tp.tail.tiles * tp.tail.parts;
    enqueue(fc_tiles<XT, WT, WM, WN, FM, FN, VEC>, dim3((unsigned)std::min<int64_t>(jobs, 1 << 22)), dim3(S::NT), 0, st, tp);
    if (size.room > 0 && (p.offsets || tp.tail.parts > 1)) start_join<XT, S::TM, S::TN>(tp, tiles, st);
}

template <int XT, int WT, bool VEC>
void run_tiles(const GroupedFc& p, const TileSize& size, float* partial, hipStream_t st) {
    if (size.rows == 32) start_tiles<XT, WT, 1, 4, 1, 1, VEC>(p, size, partial, st);
    else if constexpr (Slab<XT, WT, 2, 4, 4, 2, VEC>::kCut) start_tiles<XT, WT, 2, 4, 2, 2, VEC>(p, size, partial, st);
    else if (size.rows == 64) start_tiles<XT, WT, 1, 4, 2, 1, VEC>(p, size, partial, st);
    else if (size.outs == 128) start_tiles<XT, WT, 2, 2, 2, 2, VEC>(p, size, partial, st);
    else if constexpr (XT != CNN_MX4 && VEC) start_tiles<XT, WT, 2, 4, 4, 2, VEC>(p, size, partial, st);
}

// vec: rows of wide operands are whole 16-byte vectors.
template <int XT, int WT>
void run_tiles(const GroupedFc& p, const TileSize& size, bool vec, float* partial, hipStream_t st) {
    if (XT == CNN_MX4 || vec || Slab<XT, WT, 1, 4, 2, 1, true>::kCut) run_tiles<XT, WT, true>(p, size, partial, st);
    else if constexpr (XT != CNN_MX4 && !Slab<XT, WT, 1, 4, 2, 1, true>::kCut) run_tiles<XT, WT, false>(p, size, partial, st);
}

void run_tiles_f32(const GroupedFc&, const TileSize&, bool vec, float* partial, hipStream_t);
void run_tiles_16(const GroupedFc&, const TileSize&, bool vec, float* partial, hipStream_t);
void run_tiles_mx4(const GroupedFc&, const TileSize&, bool vec, float* partial, hipStream_t);
void run_tiles_wide_mx4(const GroupedFc&, const TileSize&, bool vec, float* partial, hipStream_t);
void run_tiles_cut(const GroupedFc&, const TileSize&, bool vec, float* partial, hipStream_t);

}  // namespace cnn
