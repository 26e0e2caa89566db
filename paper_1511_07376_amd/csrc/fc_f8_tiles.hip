// Products on 8-bit floats for many tokens: tiles of outputs x tokens, operands staged in LDS.
//
// A workgroup walks the reduction block by block.  While the matrix cores work on one, the
// next one is on its way into another LDS buffer: rows that are whole 16-byte
// vectors are copied there by the load instruction itself, other rows go through registers.
// LDS rows are a block's 128 bytes without padding (the copying loads write 64
// consecutive vectors); the vectors of a row are exchanged by an XOR with three bits of
// the row that differ between the lanes that read together.
//
// A wave's outputs are dealt to the instruction's rows so that a lane ends with 4 FO
// neighbouring outputs of a token, which it stores as they are.
//
// 2048 x 9216 x 4096 to bf16 (256 x 128 tiles): 133 to 146 us, 1.1 PFLOP/s (a large product of bf16 matrices runs
// at 1.4); the matrix cores are at work for 52% of it and the vector units, which convert both operands in every wave
// that reads them, for 57%.  64 x 9216 x 4096 to fp32 (128 x 64 tiles in 6 parts): 16 us and 4 for the join, of which reading
// the weights would take 7.5.
#include "fc_f8.h"

#include <algorithm>
#include <type_traits>

namespace cnn {
namespace {

// WO x WT waves of FO x FT fragments of 16.
template <int WO, int WT, int FO, int FT>
struct Shape {
    static constexpr int TO = WO * FO * 16, TT = WT * FT * 16, NT = 64 * WO * WT;
    static_assert(FO * 16 <= kF8Block, "a wave's outputs share their scale");
    // Exchange of a row's vectors, by three bits in which 8 neighbouring lanes' rows differ.  A lane reads vectors q and
    // q + 4 of its row (q: a quarter of the wave): 4.2 cycles a read of a wave; of 2 q and 2 q + 1 it would be 8.2.
    static __device__ int out_key(int row) { return (row & 3) | (row / (FO * 4) & 1) << 2; }
    static __device__ int token_key(int row) { return row & 7; }
};

struct TileParams {
    FcF8 fc;
    int blocks;           // of the reduction
    int out_tiles, tiles;
    int parts, run;       // parts of the reduction, blocks of each (a multiple of 4)
    bool whole_scales;    // a row's scales are whole 16-byte vectors
    float* partial;       // [parts][N][O] if parts > 1
};

// 64 lanes' 16 (4) bytes, at 32-bit offsets from a base, to consecutive places in LDS.  Not by the compiler's builtins: it
// would wait for all such copies before reads of LDS that it cannot tell from their targets, and so for those that are
// meant to be on their way while a block is worked on.  What is copied is read behind a wait and a barrier only (block_barrier).
__device__ inline unsigned lds_address(const void* p) { return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) char*)p; }
__device__ inline void copy16(const void* base, unsigned at, unsigned lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(at), "s"(base) : "m0");
}
__device__ inline void copy4(const void* base, unsigned at, unsigned lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(at), "s"(base) : "m0");
}

// One operand's vectors of a block, of this work-item: ROWS rows, NT work-items.  VEC: rows of whole blocks at
// 16-byte addresses, copied to LDS by the loads; others go through registers.  Places are
// 32-bit offsets (a tensor has fewer than 2^31 bytes) from a base that moves on with the blocks.
template <int ROWS, int NT, bool VEC, typename KEY>
struct Fetch {
    static constexpr int N = ROWS * 8 / NT;
    static_assert(ROWS * 8 % NT == 0, "whole vectors a work-item");
    unsigned at[N];
    u32x4 reg[VEC ? 1 : N];

    static __device__ int row_of(int i) { return (i * NT + (int)threadIdx.x) >> 3; }
    static __device__ int vector_of(int i) { return ((int)threadIdx.x & 7) ^ KEY::of(row_of(i)); }

    // rows beyond the last one repeat it: nothing of theirs is stored
    __device__ void begin(int64_t row0, int rows, int cols) {
#pragma unroll
        for (int i = 0; i < N; ++i) at[i] = (unsigned)min(row0 + row_of(i), (int64_t)rows - 1) * (unsigned)cols + (unsigned)(vector_of(i) * 16);
    }
    // Block k of rows of `cols` values.
    __device__ void load(const uint8_t* base, int k, int cols, char* lds) {
        base += (int64_t)k * kF8Block;
        const unsigned to = lds_address(lds) + (__builtin_amdgcn_readfirstlane((int)threadIdx.x) & ~63) * 16;  // the wave's vectors are consecutive
        const int64_t left = cols - (int64_t)k * kF8Block;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int in = vector_of(i) * 16;
            if constexpr (VEC) copy16(base, at[i], to + i * NT * 16);
            // (at odd addresses too: 1500 x 4001 x 4001 takes 99 to 103 us; loaded by words and shifted, as for few rows, it was a
            // tenth slower on products of half the time)
            else if (left >= kF8Block) reg[i] = load16(base + at[i]);
            else reg[i] = load_bytes_edge(base + at[i], left - in, (int64_t)k * kF8Block + in);
        }
    }
    __device__ void store(char* lds) {
        if constexpr (!VEC) {
#pragma unroll
            for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4*>(lds + (i * NT + (int)threadIdx.x) * 16) = reg[i];
        }
    }
};
template <typename S>
struct OutKey {
    static __device__ int of(int row) { return S::out_key(row); }
};
template <typename S>
struct TokenKey {
    static __device__ int of(int row) { return S::token_key(row); }
};

// All the wave's loads but the last LEFT have landed, its LDS accesses are done; then all waves'.
template <int LEFT = 0>
__device__ inline void block_barrier() {
    static_assert(LEFT < 64, "what the counter of loads holds");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((LEFT & 15) | LEFT >> 4 << 14 | 0x70);  // vmcnt(LEFT) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// 4 FO neighbours of a token.
template <int YT, int N>
__device__ inline void store_outputs(void* y, size_t at, const float* v, int64_t count) {
    using T = std::conditional_t<YT == CNN_F32, float, std::conditional_t<YT == CNN_BF16, bf16_t, f16_t>>;
    T* dst = (T*)y + at;
    constexpr int E = 16 / (int)sizeof(T);
#pragma unroll
    for (int h = 0; h < N / E; ++h) {
        T part[E];
#pragma unroll
        for (int c = 0; c < E; ++c) part[c] = from_f32<T>(v[h * E + c]);
        if ((h + 1) * E <= count) {
            u32x4 u;
            __builtin_memcpy(&u, part, 16);
            store16(dst + h * E, u);
        } else {
#pragma unroll
            for (int c = 0; c < E; ++c)
                if (h * E + c < count) dst[h * E + c] = part[c];
        }
    }
}

// YT: the result's type.  SPLIT: sums go to the workspace, without bias.
template <int WO, int WT, int FO, int FT, bool VEC, int YT, bool SPLIT>
__global__ void __launch_bounds__(64 * WO * WT, 2) fc_f8_tiles(TileParams tp) {
    using S = Shape<WO, WT, FO, FT>;
    constexpr int TO = S::TO, TT = S::TT, NT = S::NT;
    constexpr int kBuffer = (TO + TT) * kF8Block;
    __shared__ __attribute__((aligned(16))) char buffers[2 * kBuffer];  // outputs' rows, then tokens'
    __shared__ __attribute__((aligned(16))) float sScale[2][4 * TT];
    __shared__ float sWeight[2][64];  // the weights' scales: 4 blocks of each 128 outputs
    static_assert(NT > TT, "a lane a token, and a wave for the weights");
    const FcF8& p = tp.fc;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, quarter = lane >> 4;
    const int wo = wave / WT, wt = wave % WT, uwave = __builtin_amdgcn_readfirstlane(wave);

    const int jobs = tp.tiles * tp.parts;
    for (int turn = blockIdx.x; turn < jobs; turn += gridDim.x) {
        // Workgroups go to the eight XCDs in turn; each XCD gets a contiguous run of the jobs, so
        // that neighbours share operands in its L2.
        const int xcd = turn % 8, run = jobs / 8, more = jobs % 8;
        const int job = xcd * run + min(xcd, more) + turn / 8;
        const int part = job / tp.tiles, tile = job % tp.tiles;
        // bands of 4 tiles of tokens, walked output by output
        constexpr unsigned BAND = 4;
        const unsigned token_tiles = (unsigned)(tp.tiles / tp.out_tiles);
        const unsigned band = (unsigned)tile / (BAND * (unsigned)tp.out_tiles), in_band = (unsigned)tile % (BAND * (unsigned)tp.out_tiles);
        const unsigned band_rows = min(BAND, token_tiles - band * BAND);
        const int64_t o0 = (int64_t)(in_band / band_rows) * TO, n0 = (int64_t)(band * BAND + in_band % band_rows) * TT;
        const int first = part * tp.run, last = min(first + tp.run, tp.blocks);

        Fetch<TO, NT, VEC, OutKey<S>> fw;
        Fetch<TT, NT, VEC, TokenKey<S>> fx;
        fw.begin(o0, p.O, p.I);
        fx.begin(n0, p.N, p.I);
        // The inputs' scales come in groups of 4 blocks, a lane a token: a row's are neighbours, and a line for
        // every token and block would take as long as the operands (2048 x 9216 x 4096 on products of half the time:
        // 99 us against 109 with half as many of them, and 77 against 100 for the copies alone).  So do the weights', a lane one of them.  (A scalar load of
        // the block's would make the reads of LDS after it wait for all before.)
        const unsigned xs = (unsigned)min(tid % TT, (int)min((int64_t)p.N - 1 - n0, (int64_t)TT)) * (unsigned)tp.blocks * 4;  // fewer than 2^31 bytes
        auto ask_scales = [&](int group) {
            const int k = first + 4 * group;
            if (uwave == TT / 64) {
                const unsigned row = (unsigned)min((o0 >> 7) + (lane >> 2), (int64_t)(p.O - 1) >> 7);
                copy4(p.ws, (row * (unsigned)tp.blocks + (unsigned)min(k + (lane & 3), tp.blocks - 1)) * 4, lds_address(sWeight[group & 1]));
            }
            if (uwave >= TT / 64) return;
            const float* base = p.xs + (size_t)n0 * tp.blocks;
            const unsigned dst = lds_address(sScale[group & 1]);
            if (tp.whole_scales) {
                copy16(base + k, xs, dst + uwave * 64 * 16);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) copy4(base + min(k + i, tp.blocks - 1), xs, dst + (i * TT + uwave * 64) * 4);
            }
        };
        const int scale_token = tp.whole_scales ? 4 : 1, scale_block = tp.whole_scales ? 1 : TT;

        f32x4 acc[FO][FT];
#pragma unroll
        for (int i = 0; i < FO; ++i)
#pragma unroll
            for (int j = 0; j < FT; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

        // Rows of fragment f: (l16 / 4) 4 FO + 4 f + l16 % 4 of the outputs, 16 f + l16 of the tokens.
        const int orow = wo * FO * 16 + (l16 >> 2) * (FO * 4) + (l16 & 3), trow = wt * FT * 16 + l16;
        auto read = [&](const char* base, int row, int key) {
            const int v = quarter ^ key;
            return Bytes{*reinterpret_cast<const u32x4*>(base + row * kF8Block + v * 16),
                         *reinterpret_cast<const u32x4*>(base + row * kF8Block + (v ^ 4) * 16)};
        };
        // Asks for block k, or, behind the last one, for that again (nothing comes of it).
        auto ask = [&](int k, char* to) {
            k = min(k, last - 1);
            fw.load(p.w, k, p.I, to);
            fx.load(p.x, k, p.I, to + TO * kF8Block);
        };
        const int key = S::out_key(orow);
        Halves x[FT];
        Bytes next;                   // the outputs' next fragment
        f32x4 d[2][FT];               // a fragment's sums, and those of the one before
        float s[FT], before[FT];      // a block's scales, and those of the one before
        auto read_scales = [&](int k, float* to) {
            const int at = k - first;
            const float w = sWeight[(at >> 2) & 1][(wo * FO * 16 >> 7) * 4 + (at & 3)];
            const float* group = sScale[(at >> 2) & 1] + (at & 3) * scale_block + trow * scale_token;
#pragma unroll
            for (int j = 0; j < FT; ++j) {
                const float v = group[16 * j * scale_token] * w;
                to[j] = k < last ? v : 0.0f;
            }
        };
        auto read_token = [&](const char* buffer, int j) { x[j] = to_halves(read(buffer + TO * kF8Block, trow + 16 * j, S::token_key(l16))); };
        // Block k, whose first fragments are in registers.  The products of a fragment of outputs are at work while the sums
        // of the one before are added.  Before its last fragment's products the next block is made ready, the one after it is
        // asked for (this one's buffer is free: all waves have read what they need), and the next one's
        // first fragments are read: those products cover that.
        auto work = [&](int k, char* here, char* after) {
            float s_after[FT];
#pragma unroll
            for (int i = 0; i < FO; ++i) {
                const Halves w = to_halves(next);
                if (i + 1 < FO) {
                    next = read(here, orow + 4 * (i + 1), key);
                } else {
                    fw.store(after);
                    fx.store(after + TO * kF8Block);
                    block_barrier();
                    read_scales(k + 1, s_after);
                    next = read(after, orow, key);
                    __builtin_amdgcn_sched_barrier(0);
                    ask(k + 2, here);
                    // the other group's places have been read by all waves; what is asked for now is used 3 blocks later,
                    // behind the barriers between, which wait for it
                    if (((k - first) & 3) == 0 && k + 4 < last) ask_scales(((k - first) >> 2) + 1);
                }
#pragma unroll
                for (int j = 0; j < FT; ++j) {
                    d[i % 2][j] = block_sums(w, x[j]);
                    if (i + 1 == FO) read_token(after, j);
                    const int done = (i + FO - 1) % FO;
                    add_scaled(acc[done][j], d[(i + 1) % 2][j], i == 0 ? before[j] : s[j]);
                    asm volatile("" : "+v"(acc[done][j]));  // here, and not when the sum is next needed
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
#pragma unroll
            for (int j = 0; j < FT; ++j) before[j] = s[j], s[j] = s_after[j];
        };
        static_assert(FO % 2 == 0, "a fragment's set of sums is the same in every block");
        if (first < last) {
            ask_scales(0);
            ask(first, buffers);
            fw.store(buffers);
            fx.store(buffers + TO * kF8Block);
            ask(first + 1, buffers + kBuffer);
            block_barrier<VEC ? decltype(fw)::N + decltype(fx)::N : 0>();  // that block's loads may be on their way
            next = read(buffers, orow, key);
            read_scales(first, s);
#pragma unroll
            for (int j = 0; j < FT; ++j) {
                read_token(buffers, j);
                before[j] = 0.0f;
                d[1][j] = f32x4{0, 0, 0, 0};
            }
            // whole turns of the buffers: a block behind the last one has a scale of 0
#pragma unroll 1
            for (int k = first; k < last; k += 2) {
                work(k, buffers, buffers + kBuffer);
                work(k + 1, buffers + kBuffer, buffers);
            }
#pragma unroll
            for (int j = 0; j < FT; ++j) add_scaled(acc[FO - 1][j], d[1][j], before[j]);
        }

        const int64_t o = o0 + wo * FO * 16 + quarter * (FO * 4), count = min((int64_t)p.O - o, (int64_t)FO * 4);
        if (count > 0) {
            float bias[FO * 4];
#pragma unroll
            for (int c = 0; c < FO * 4; ++c) bias[c] = !SPLIT && p.bias && c < count ? p.bias[o + c] : 0.0f;
#pragma unroll
            for (int j = 0; j < FT; ++j) {
                const int64_t n = n0 + (wt * FT + j) * 16 + l16;
                if (n >= p.N) continue;
                float v[FO * 4];
#pragma unroll
                for (int c = 0; c < FO * 4; ++c) v[c] = SPLIT ? acc[c / 4][j][c % 4] : finish(p, acc[c / 4][j][c % 4], bias[c]);
                if constexpr (SPLIT) store_outputs<CNN_F32, FO * 4>(tp.partial + (size_t)part * p.N * p.O, (size_t)n * p.O + o, v, count);
                else store_outputs<YT, FO * 4>(p.y, (size_t)n * p.O + o, v, count);
            }
        }
        block_barrier();  // nothing is on its way to the buffers, which are the next tile's
    }
}

// Adds the parts of a split reduction, in their order, then bias and ReLU: 4 neighbours a work-item.
template <int YT>
__global__ void __launch_bounds__(256) fc_f8_join(TileParams tp) {
    const FcF8& p = tp.fc;
    const int64_t all = (int64_t)p.N * p.O, step = (int64_t)gridDim.x * 1024;
    for (int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; e < all; e += step) {
        const int count = (int)min(all - e, (int64_t)4);
        float v[4] = {0, 0, 0, 0};
#pragma unroll 4
        for (int q = 0; q < tp.parts; ++q) {
            const float* src = tp.partial + (size_t)q * all + e;
            if (count == 4) {
                f32x4 u;
                __builtin_memcpy(&u, src, 16);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] += u[i];
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (i < count) v[i] += src[i];
            }
        }
        int o = (int)(e % p.O);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = finish(p, v[i], p.bias && i < count ? p.bias[o] : 0.0f);
            o = o + 1 == p.O ? 0 : o + 1;
        }
        if constexpr (YT == CNN_F32) {
            store_outputs<YT, 4>(p.y, (size_t)e, v, count);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < count) store_value(YT, p.y, (size_t)e + i, v[i]);
        }
    }
}

template <int WO, int WT, int FO, int FT, bool VEC, int YT>
void start(const FcF8& p, const F8Tile& t, float* partial, hipStream_t st) {
    using S = Shape<WO, WT, FO, FT>;
    const int blocks = f8_blocks(p.I);
    TileParams tp{p, blocks, ceil_div(p.O, S::TO), 0, t.parts, t.run, (uintptr_t)p.xs % 16 == 0 && blocks % 4 == 0, partial};
    tp.tiles = tp.out_tiles * ceil_div(p.N, S::TT);
    const dim3 grid((unsigned)std::min<int64_t>((int64_t)tp.tiles * tp.parts, 1 << 20));
    if (t.parts == 1) {
        enqueue(fc_f8_tiles<WO, WT, FO, FT, VEC, YT, false>, grid, dim3(S::NT), 0, st, tp);
    } else {
        enqueue(fc_f8_tiles<WO, WT, FO, FT, VEC, YT, true>, grid, dim3(S::NT), 0, st, tp);
        enqueue(fc_f8_join<YT>, dim3((unsigned)std::min<int64_t>(ceil_div64((int64_t)p.N * p.O, 1024), 1 << 16)), dim3(256), 0, st, tp);
    }
}

template <int WO, int WT, int FO, int FT, bool VEC>
void start_type(const FcF8& p, const F8Tile& t, float* partial, hipStream_t st) {
    if (p.y_type == CNN_F32) {
        start<WO, WT, FO, FT, VEC, CNN_F32>(p, t, partial, st);
    } else if (p.y_type == CNN_BF16) {
        start<WO, WT, FO, FT, VEC, CNN_BF16>(p, t, partial, st);
    } else {
        start<WO, WT, FO, FT, VEC, CNN_F16>(p, t, partial, st);
    }
}

}  // namespace

void run_f8_tiles(const FcF8& p, const F8Tile& t, bool vec, float* partial, hipStream_t st) {
    if (t.tokens == 64) {
        if (vec) start_type<2, 2, 4, 2, true>(p, t, partial, st);
        else start_type<2, 2, 4, 2, false>(p, t, partial, st);
    } else if (t.outs == 128) {
        if (vec) start_type<2, 2, 4, 4, true>(p, t, partial, st);
        else start_type<2, 2, 4, 4, false>(p, t, partial, st);
    } else {
        start_type<4, 2, 4, 4, true>(p, t, partial, st);
    }
}

}  // namespace cnn
