// Products on 8-bit floats for many tokens: tiles of outputs x tokens, operands staged in LDS.
//
// A workgroup walks the reduction block by block.  While the matrix cores work on one, the
// next one is on its way into the other LDS buffer: rows that are whole 16-byte vectors
// are copied there by the load instruction itself, other rows go through registers.
// LDS rows are a block's 128 bytes without padding (the copying loads write 64
// consecutive vectors); the vectors of a row are exchanged by an XOR with three bits of
// the row that differ between the lanes that read together.
//
// A wave's outputs are dealt to the instruction's rows so that a lane ends with 4 FO
// neighbouring outputs of a token, which it stores as they are.
#include "fc_f8.h"

#include <algorithm>
#include <type_traits>

namespace cnn {
namespace {

static __device__ const u32x4 kZeroVector = {0, 0, 0, 0};

// WO x WT waves of FO x FT fragments of 16.
template <int WO, int WT, int FO, int FT>
struct Shape {
    static constexpr int TO = WO * FO * 16, TT = WT * FT * 16, NT = 64 * WO * WT;
    static_assert(FO * 16 <= kF8Block, "a wave's outputs share their scale");
    // exchange of a row's vectors
    static __device__ int out_key(int row) { return (row & 3) | ((row / (FO * 4)) & 1) << 2; }
    static __device__ int token_key(int row) { return row & 7; }
};

struct TileParams {
    FcF8 fc;
    int blocks;           // of the reduction
    int out_tiles, tiles;
    int parts, run;       // parts of the reduction, blocks of each
    float* partial;       // [parts][N][O] if parts > 1
};

__device__ inline void copy16(const uint8_t* src, char* dst) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                     (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}

// One operand's vectors of a block, of this work-item: ROWS rows, NT work-items.  Places are
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
    // Block k of rows of `cols` values.  FULL: all of it is in them.
    template <bool FULL>
    __device__ void load(const uint8_t* base, int k, int cols, char* lds) {
        base += (int64_t)k * kF8Block;
        const int64_t left = cols - (int64_t)k * kF8Block;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int in = vector_of(i) * 16;
            if constexpr (VEC) copy16(FULL || in < left ? base + at[i] : (const uint8_t*)&kZeroVector, lds + (i * NT + (int)(threadIdx.x & ~63u)) * 16);
            else if (FULL || left >= kF8Block) reg[i] = load16(base + at[i]);
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

// All loads of the wave have landed, its LDS accesses are done; then all waves'.
__device__ inline void block_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x70);  // vmcnt(0) lgkmcnt(0)
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

// YT: the result's type; fp32 ones are summed in 16 bits, others on the 8-bit instruction.
// SPLIT: sums go to the workspace, without bias.
template <int WO, int WT, int FO, int FT, bool VEC, int YT, bool SPLIT>
__global__ void __launch_bounds__(64 * WO * WT, 2) fc_f8_tiles(TileParams tp) {
    using S = Shape<WO, WT, FO, FT>;
    using Operand = std::conditional_t<YT == CNN_F32, Halves, Bytes>;
    constexpr int TO = S::TO, TT = S::TT, NT = S::NT;
    // arrays of their own: the compiler sees that a copy into one does not concern reads of another
    __shared__ __attribute__((aligned(16))) char sW0[TO * kF8Block], sW1[TO * kF8Block], sX0[TT * kF8Block], sX1[TT * kF8Block];
    const FcF8& p = tp.fc;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, quarter = lane >> 4;
    const int wo = wave / WT, wt = wave % WT;

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
        const float* ws = p.ws + (size_t)min((o0 + wo * FO * 16) >> 7, (int64_t)(p.O - 1) >> 7) * tp.blocks;
        unsigned xs[FT];
#pragma unroll
        for (int j = 0; j < FT; ++j) xs[j] = (unsigned)min(n0 + (wt * FT + j) * 16 + l16, (int64_t)p.N - 1) * (unsigned)tp.blocks;
        float wnext = 0, xnext[FT];
        auto load_scales = [&](int k) {
            wnext = ws[k];
#pragma unroll
            for (int j = 0; j < FT; ++j) xnext[j] = (p.xs + k)[xs[j]];
        };

        f32x4 acc[FO][FT];
#pragma unroll
        for (int i = 0; i < FO; ++i)
#pragma unroll
            for (int j = 0; j < FT; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

        // Rows of fragment f: (l16 / 4) 4 FO + 4 f + l16 % 4 of the outputs, 16 f + l16 of the tokens.
        const int orow = wo * FO * 16 + (l16 >> 2) * (FO * 4) + (l16 & 3), trow = wt * FT * 16 + l16;
        // a lane's first vector of a fragment, 2 quarter; the second is an XOR with 1 away
        auto read = [&](const char* base, int row, int key) {
            const int v = (2 * quarter) ^ key;
            return Bytes{*reinterpret_cast<const u32x4*>(base + row * kF8Block + v * 16),
                         *reinterpret_cast<const u32x4*>(base + row * kF8Block + (v ^ 1) * 16)};
        };
        auto as_operand = [&](const Bytes& b) {
            if constexpr (YT == CNN_F32) return to_halves(b);
            else return b;
        };
        // The products of a fragment of outputs are at work while the sums of the one before are added.
        auto multiply = [&](const char* W, const char* X, const float* s) {
            Operand x[FT];
#pragma unroll
            for (int j = 0; j < FT; ++j) x[j] = as_operand(read(X, trow + 16 * j, S::token_key(l16)));
            const int key = S::out_key(orow);
            Bytes next = read(W, orow, key);
            f32x4 d[2][FT];
#pragma unroll
            for (int i = 0; i <= FO; ++i) {
                if (i < FO) {
                    const Operand w = as_operand(next);
                    if (i + 1 < FO) next = read(W, orow + 4 * (i + 1), key);
#pragma unroll
                    for (int j = 0; j < FT; ++j) d[i % 2][j] = block_sums(w, x[j]);
                }
                if (i > 0) {
#pragma unroll
                    for (int j = 0; j < FT; ++j) {
                        add_scaled(acc[i - 1][j], d[(i - 1) % 2][j], s[j]);
                        asm volatile("" : "+v"(acc[i - 1][j]));  // here, and not when the sum is next needed
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // Block k, which is in (W, X) or on its way there; the next one goes to (NW, NX).
        auto work = [&](int k, auto full, const char* W, const char* X, char* NW, char* NX) {
            constexpr bool FULL = decltype(full)::value;  // there is a next one, a whole one
            block_barrier();
            float s[FT];
#pragma unroll
            for (int j = 0; j < FT; ++j) s[j] = xnext[j] * wnext;
            if (FULL || k + 1 < last) {
                fw.template load<FULL>(p.w, k + 1, p.I, NW);
                fx.template load<FULL>(p.x, k + 1, p.I, NX);
                load_scales(k + 1);
            }
            multiply(W, X, s);
            if (FULL || k + 1 < last) {
                fw.store(NW);
                fx.store(NX);
            }
        };
        if (first < last) {
            fw.template load<false>(p.w, first, p.I, sW0);
            fx.template load<false>(p.x, first, p.I, sX0);
            load_scales(first);
            fw.store(sW0);
            fx.store(sX0);
            int k = first;
            for (; k + 3 < last; k += 2) {
                work(k, std::true_type{}, sW0, sX0, sW1, sX1);
                work(k + 1, std::true_type{}, sW1, sX1, sW0, sX0);
            }
            for (; k < last; k += 2) {
                work(k, std::false_type{}, sW0, sX0, sW1, sX1);
                if (k + 1 < last) work(k + 1, std::false_type{}, sW1, sX1, sW0, sX0);
            }
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
        __syncthreads();  // the buffers are the next tile's
    }
}

template <int WO, int WT, int FO, int FT, bool VEC, int YT, bool SPLIT>
void start(const TileParams& tp, hipStream_t st) {
    using S = Shape<WO, WT, FO, FT>;
    const int64_t jobs = (int64_t)tp.tiles * tp.parts;
    enqueue(fc_f8_tiles<WO, WT, FO, FT, VEC, YT, SPLIT>, dim3((unsigned)std::min<int64_t>(jobs, 1 << 20)), dim3(S::NT), 0, st, tp);
}

template <int WO, int WT, int FO, int FT, bool VEC>
void start_type(const FcF8& p, const F8Tile& t, float* partial, hipStream_t st) {
    using S = Shape<WO, WT, FO, FT>;
    const int blocks = f8_blocks(p.I);
    TileParams tp{p, blocks, ceil_div(p.O, S::TO), 0, 1, blocks, partial};
    tp.tiles = tp.out_tiles * ceil_div(p.N, S::TT);
    if (p.y_type == CNN_F32) start<WO, WT, FO, FT, VEC, CNN_F32, false>(tp, st);
    else if (p.y_type == CNN_BF16) start<WO, WT, FO, FT, VEC, CNN_BF16, false>(tp, st);
    else start<WO, WT, FO, FT, VEC, CNN_F16, false>(tp, st);
}

}  // namespace

void run_f8_tiles(const FcF8& p, const F8Tile& t, bool vec, float* partial, hipStream_t st) {
    if (t.outs == 256 && vec && p.y_type != CNN_F32) start_type<2, 4, 8, 4, true>(p, t, partial, st);
    else if (vec) start_type<2, 2, 4, 4, true>(p, t, partial, st);
    else start_type<2, 2, 4, 4, false>(p, t, partial, st);
}

}  // namespace cnn
