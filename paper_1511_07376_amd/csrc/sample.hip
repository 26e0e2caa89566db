// A token for each row of logits: temperature, top-k, top-p, min-p, then the token that a
// random number of the caller's falls on.
//
// Which token that is, and where top-p ends, is a matter of sums next to a border, so
// weights exp((l - max l) / T) are taken as whole numbers of 2^-S of the largest (S = 51, less
// where 2^S times V would pass 64 bits) from an exponential in 64-bit floats.  Their sums
// are exact, whatever the order: additions can be atomic, split, and done twice with
// the same result.
//
// Rows are not sorted.  The tokens' order (falling logit, rising number) is a code of 64 bits
// for each, and the last token that a rule keeps is the one at which a count (top-k) or a
// sum (top-p) is reached: it is found by histograms, first over bins of equal width in log2 of
// the weight, then over the digits of the codes of the tokens in the bin where the
// border lies.  The draw is the same search over the tokens' numbers, whose first bins are
// tiles of the row.  Once all that a row keeps fits a list in LDS, the rest is done there; by
// sorting it after all where that is no more than a token a work-item.
//
// One workgroup does a row, or, where there are few long rows, several do what passes over all
// of it: the largest logit, the first histogram, the list, the tiles' sums.
//
// Not bound by memory.  256 rows of 50021 fp16, a temperature alone: 29 us, 0.9 TB/s, in which some 50 instructions a
// logit are issued, half of them the 64-bit exponential: the vector units are at work for 62% of the time, waves wait for
// loads and each other at barriers for the rest (loading further ahead changed nothing).  64 rows of
// 131072 bf16 with all the rules: 70 us, the six kernels taking 6 (largest), 15 (bins), 12 (list), 13
// (cuts), 9 (tiles), 8 (draw), of which each one's start and end is about 3.  7 rows of 1000: 12 us, a chain of
// barriers.
//
#include "f8.h"

#include <algorithm>
#include <type_traits>

namespace cnn {
namespace {

typedef unsigned long long u64;

constexpr int kBins = 2048;
constexpr float kBinsPerOctave = 38.0f;  // the last bin begins at 2^-53.8, which is no whole number's weight
constexpr int kDigit = 8, kDigits = 1 << kDigit;
constexpr int kFew = 64;                // tokens that a wave finishes a search among
constexpr int kList = 2048;             // tokens that are worked on in LDS
constexpr u64 kAll = ~0ull;

#define CNN_INLINE __device__ inline __attribute__((always_inline))

// What a row shares between the kernels of a call that splits rows.
struct Split {
    u64* best;      // [N][chunks] largest logit and its first token, of a chunk
    u64* last;      // [N] code of the last token kept
    u64* list;      // [N][kList] codes
    int* listed;    // [N]
    int* pending;   // [N] whether the draw is still to be made
    u64* sum;       // [N][kBins]
    unsigned* count;  // [N][kBins]
    int chunks, chunk;  // 0 chunks: rows are not split
};
struct Args {
    Sample p;
    int bits;  // S
    int each;  // tokens of a tile
    Split split;
};

// ---------------------------------------------------------------- a row
// What a row's logits are compared and weighed by.
struct Scale {
    float top;     // the largest logit; 0 where that is infinite
    bool infinite;  // then the infinite ones are 0, the others are none
    double per;    // log2(e) / T
    float bins;    // bins two units of the logits
    int bits;
    // A logit as it counts: minus infinity is none.  -0 becomes +0.
    CNN_INLINE float value(float l) const {
        if (infinite) return l == INFINITY ? 0.0f : -INFINITY;
        return l > -INFINITY ? l + 0.0f : -INFINITY;
    }
    // Not falling as the logit falls, in the same way wherever it is called; the last one for minus infinity and NaN.
    // (Halves: the difference of the largest and the least float is more than a float.)
    CNN_INLINE int bin(float v) const { return (int)fminf((0.5f * top - 0.5f * v) * bins, (float)(kBins - 1)); }
    // 2^bits exp((v - top) / T), rounded to a whole number: 2^f by a polynomial that
    // interpolates it at the Chebyshev nodes of [-1/2, 1/2] (to 3e-16), 1 at f = 0.
    CNN_INLINE u64 weight(float v) const {
        const double t = fmax(((double)v - (double)top) * per, -100.0);
        const double n = __builtin_rint(t), f = t - n;
        double w = 0x1.e6063f7217bc6p-28;
        w = fma(w, f, 0x1.b675bca4eeebbp-24);
        w = fma(w, f, 0x1.62bfd47773353p-20);
        w = fma(w, f, 0x1.ffcb54062e698p-17);
        w = fma(w, f, 0x1.430913096fd9fp-13);
        w = fma(w, f, 0x1.5d87fe9d7a584p-10);
        w = fma(w, f, 0x1.3b2ab6fba1ddap-7);
        w = fma(w, f, 0x1.c6b08d703ce49p-5);
        w = fma(w, f, 0x1.ebfbdff82c598p-3);
        w = fma(w, f, 0x1.62e42fefa3a19p-1);
        w = fma(w, f, 1.0);
        // 2^52 more, and the whole number stands in the low bits
        w = __builtin_ldexp(w, (int)n + bits) + 0x1p52;
        return (u64)__double_as_longlong(w) & 0x000fffffffffffffull;
    }
};

// Rises with the logit.
CNN_INLINE unsigned key_of(float v) {
    const unsigned b = __float_as_uint(v);
    return b >> 31 ? ~b : b | 0x80000000u;
}
// The order of the tokens: falling logit, rising number.
CNN_INLINE u64 code_of(float v, int i) { return (u64)~key_of(v) << 32 | (unsigned)i; }

CNN_INLINE float value_of(u64 code) {
    const unsigned k = ~(unsigned)(code >> 32);
    return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k);
}

struct Parameters {
    float u, temperature, top_p, min_p;
    int top_k;
    CNN_INLINE Parameters(const Sample& p, int row)
        : u(p.u[row]), temperature(p.temperature ? p.temperature[row] : 1.0f), top_p(p.top_p ? p.top_p[row] : 1.0f),
          min_p(p.min_p ? p.min_p[row] : 0.0f), top_k(p.top_k ? p.top_k[row] : 0) {}
};

// What follows from a row's parameters and its largest logit.
struct Row {
    float u, top_p;
    int top_k, first;
    bool cut_k, cut_p;
    u64 least;       // the least weight that min-p keeps
    u64 first_code;
    Scale scale;
    int token;       // -2: to be drawn
    float prob;
    // best: the largest logit's key and the complement of its first token; 0: there is none
    CNN_INLINE Row(const Args& a, const Parameters& q, u64 best) {
        u = q.u;
        top_p = q.top_p;
        top_k = q.top_k;
        first = (int)~(unsigned)best;
        token = -2;
        prob = 1.0f;
        const bool fine = q.temperature >= 0.0f && q.temperature < INFINITY && u == u && top_p == top_p && q.min_p == q.min_p;
        if (best == 0 || !fine) token = -1, prob = 0.0f;
        else if (q.temperature == 0.0f || top_k == 1 || top_p <= 0.0f || q.min_p > 1.0f) token = first;
        const float most = value_of((u64)~(unsigned)(best >> 32) << 32);
        scale.infinite = most == INFINITY;
        scale.top = scale.infinite ? 0.0f : most;
        scale.per = 1.4426950408889634 / (double)q.temperature;
        scale.bins = (float)fmin(2.0 * scale.per * (double)kBinsPerOctave, 3e38);
        scale.bits = a.bits;
        first_code = code_of(scale.top, first);
        cut_k = top_k > 0 && top_k < a.p.V;
        cut_p = top_p < 1.0f;
        least = q.min_p > 0.0f ? (u64)__builtin_ceil((double)fminf(q.min_p, 1.0f) * (double)(1ull << a.bits)) : 0;
    }
    CNN_INLINE bool keeps(u64 code, u64 w, u64 last) const { return code <= last && (w >= least || code == first_code); }
};

// f(token, 8 logits from it on) for the tokens from `from` to `to` of a row of V, 8 neighbours a work-item (`from` is a
// multiple of 8).  Logits of no token are minus infinity.
template <typename T>
CNN_INLINE void load_logits(const T* row, int64_t c, int64_t to, int V, float* v) {
    load_values8(row, (int)c, V, v);
    if (to - c < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < to ? v[i] : -INFINITY;
    }
}
template <typename T, typename F>
CNN_INLINE void each_eight(const T* row, int64_t from, int64_t to, int V, F&& f) {
    for (int64_t c = from + threadIdx.x * 8; c < to; c += (int64_t)blockDim.x * 8) {
        float v[8];
        load_logits(row, c, to, V, v);
        f((int)c, v);
    }
}
// f(token, logit) for each.
template <typename T, typename F>
CNN_INLINE void each_logit(const T* row, int64_t from, int64_t to, int V, F&& f) {
    each_eight(row, from, to, V, [&](int c, const float* v) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f(c + i, v[i]);
    });
}

// ---------------------------------------------------------------- within a workgroup
// NT work-items.
template <int NT>
struct Shared {
    static constexpr int kWaves = NT / 64;
    u64 sum[kBins];
    unsigned count[kBins];
    // digits of codes; all 0 between searches
    u64 digit_sum[kDigits];
    unsigned digit_count[kDigits];
    u64 few_code[kFew], few_weight[kFew];
    u64 wave_sum[kWaves];
    unsigned wave_count[kWaves];
    int few;
    u64 found_sum, found_code;
    unsigned found_count, found_many;
    int found;
    int listed;
};
struct List {
    u64 weight[kList];
    u64 code[kList];
};

// The value that a lane's neighbour by a data-parallel move has, 0 where there is none.
template <int CTRL, int ROWS>
CNN_INLINE unsigned moved(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false); }
template <int CTRL, int ROWS>
CNN_INLINE u64 moved(u64 v) { return (u64)moved<CTRL, ROWS>((unsigned)(v >> 32)) << 32 | moved<CTRL, ROWS>((unsigned)v); }
// op over the lanes up to and with each (0 is its neutral element): shifts by 1, 2, 4, 8 within rows of 16, then
// the rows before.
template <typename U, typename OP>
CNN_INLINE U wave_scan(U v, OP&& op) {
    v = op(v, moved<0x111, 0xf>(v));
    v = op(v, moved<0x112, 0xf>(v));
    v = op(v, moved<0x114, 0xf>(v));
    v = op(v, moved<0x118, 0xf>(v));
    v = op(v, moved<0x142, 0xa>(v));
    return op(v, moved<0x143, 0xc>(v));
}
template <typename U>
CNN_INLINE U wave_scan(U v) { return wave_scan(v, [](U a, U b) { return a + b; }); }
CNN_INLINE u64 last_lane(u64 v) {
    return (u64)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), 63) << 32 | (unsigned)__builtin_amdgcn_readlane((int)v, 63);
}
CNN_INLINE u64 wave_sum(u64 v) { return last_lane(wave_scan(v)); }
CNN_INLINE u64 wave_max(u64 v) { return last_lane(wave_scan(v, [](u64 a, u64 b) { return max(a, b); })); }

// op over the waves' values, in every work-item.
template <int NT, typename OP>
CNN_INLINE u64 over_waves(Shared<NT>& s, u64 v, OP&& op) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.wave_sum[threadIdx.x >> 6] = v;
    __syncthreads();
    v = s.wave_sum[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) v = op(v, s.wave_sum[w]);
    return v;
}
template <int NT>
CNN_INLINE u64 group_sum(Shared<NT>& s, u64 v) { return over_waves(s, wave_sum(v), [](u64 a, u64 b) { return a + b; }); }
template <int NT>
CNN_INLINE u64 group_max(Shared<NT>& s, u64 v) { return over_waves(s, wave_max(v), [](u64 a, u64 b) { return max(a, b); }); }

// The sums of the work-items up to and with each, over the workgroup; `all`: that of all.
template <int NT>
CNN_INLINE u64 group_scan(Shared<NT>& s, u64 w, u64& all) {
    const int wave = threadIdx.x >> 6;
    w = wave_scan(w);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) s.wave_sum[wave] = w;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int v = 0; v < NT / 64; ++v) {
        const u64 other = s.wave_sum[v];
        all += other;
        w += v < wave ? other : 0;
    }
    return w;
}

template <int NT>
CNN_INLINE void clear_bins(Shared<NT>& s) {
#pragma unroll
    for (int i = threadIdx.x; i < kBins; i += NT) s.sum[i] = 0, s.count[i] = 0;
    __syncthreads();
}

// ---------------------------------------------------------------- searches
// A border: the first place at which the tokens up to and with it are `count`, or
// weigh `share` or more, or weigh more than `beyond`.
enum Kind { COUNT, SHARE, DRAW };
struct Border {
    int kind;
    u64 count;
    double share;
    u64 beyond;
    CNN_INLINE bool reached(u64 c, u64 w) const {
        return kind == COUNT ? c >= count : kind == SHARE ? (double)w >= share : w > beyond;
    }
};
struct Place {
    int bin;     // -1: nowhere
    u64 count;   // tokens before the bin, and their weight
    u64 sum;
    unsigned many;  // tokens in the bin
};

// Of a work-item's N bins from `at` on, which hold (c, w) behind (count, sum): writes down the one in which the
// border lies.  Before the bins it is not reached, behind them it is: so in one work-item only.  (A
// border that nothing reaches is at the first token: none stands before it.)
template <int N, int NT>
CNN_INLINE void find_among(Shared<NT>& s, const Border& b, const u64* sums, const unsigned* counts, int at, u64 count, u64 sum, unsigned c, u64 w, u64 none) {
    if (c == 0 || (count > none && b.reached(count, sum)) || !b.reached(count + c, sum + w)) return;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (counts[i] > 0 && b.reached(count + counts[i], sum + sums[i])) {
            s.found = at + i;
            s.found_sum = sum;
            s.found_count = (unsigned)count;
            s.found_many = counts[i];
            return;
        }
        sum += sums[i], count += counts[i];
    }
}

// The first bin in which the border lies.  The bins are complete (a barrier behind them).
template <int NT>
CNN_INLINE Place find_bin(Shared<NT>& s, const Border& b) {
    constexpr int N = kBins / NT;  // bins a work-item
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = threadIdx.x * N;
    u64 sums[N], w = 0;
    unsigned counts[N], c = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) w += sums[i] = s.sum[at + i], c += counts[i] = s.count[at + i];
    const u64 win = wave_scan(w);
    const unsigned cin = wave_scan(c);
    __syncthreads();
    if (threadIdx.x == 0) s.found = -1;
    if (lane == 63) s.wave_sum[wave] = win, s.wave_count[wave] = cin;
    __syncthreads();
    u64 sum = win - w, count = cin - c;
#pragma unroll
    for (int v = 0; v < NT / 64; ++v) {
        sum += v < wave ? s.wave_sum[v] : 0;
        count += v < wave ? s.wave_count[v] : 0;
    }
    find_among<N>(s, b, sums, counts, at, count, sum, c, w, 0);
    __syncthreads();
    const Place p{s.found, s.found_count, s.found_sum, s.found_many};
    __syncthreads();
    return p;
}

// The tokens that a search is among: those of the list, or those of the row in one bin.  Of them
// the ones that are kept.
template <typename T>
struct Items {
    const T* x;
    int V;
    const Row& r;
    const List& list;
    int listed;  // -1: the row's
    int kind, bin;
    u64 last;
    // f(code, weight); the code is the token's number in a draw
    template <typename F>
    CNN_INLINE void go(F&& f) const {
        if (listed >= 0) {
#pragma unroll 1
            for (int i = threadIdx.x; i < listed; i += blockDim.x) {
                const u64 code = list.code[i], w = list.weight[i];
                if (kind != DRAW ? code <= last : r.keeps(code, w, last)) f(kind == DRAW ? code & 0xffffffffu : code, w);
            }
        } else {
            // slow: more tokens in a bin than the list holds.  16-bit logits that are coarser than a bin come here: 64 rows
            // of 131072 bf16, normal around 10 to 40 and cut by top-p 0.95, take 330 to 355 us where they take 82 around 0
#pragma unroll 1
            for (int64_t i = threadIdx.x; i < V; i += blockDim.x) {
                const float v = r.scale.value(to_f32(x[i]));
                if (v == -INFINITY || r.scale.bin(v) != bin) continue;
                const u64 code = code_of(v, (int)i);
                if (code <= last) f(code, kind == COUNT ? 0 : r.scale.weight(v));
            }
        }
    }
};

// The first code, of the items' in rising order, at which the border is reached: there is one.  Before
// all of the items: (none, sum).  `weight`: the found one's.
//
// Digit by digit from the top one that differs, one wave looking through a digit's 256 sums, until a few items
// are left: those before each are added up.
template <int NT, typename T>
CNN_INLINE u64 find_code(Shared<NT>& s, const Items<T>& items, const Border& b, u64 none, u64 sum, u64& weight) {
    u64 low = kAll, high = 0;
    items.go([&](u64 code, u64) { low = min(low, code), high = max(high, code); });
    low = ~group_max(s, ~low);
    const u64 range = group_max(s, high) - low;
    int shift = range == 0 ? 0 : max(64 - __builtin_clzll(range) - kDigit, 0);
    u64 prefix = 0, count = none;  // prefix: of what is behind low, its digits so far; lower ones 0
    int above = 64;  // bits from here on are the prefix's
#pragma unroll 1
    for (;;) {
        items.go([&](u64 code, u64 w) {
            const u64 rel = code - low;
            if (above < 64 && rel >> above != prefix >> above) return;
            const int digit = (int)(rel >> shift) & (kDigits - 1);
            atomicAdd(&s.digit_sum[digit], w);
            atomicAdd(&s.digit_count[digit], 1u);
        });
        if (threadIdx.x == 0) s.found = -1;
        __syncthreads();
        if (threadIdx.x < 64) {
            constexpr int N = kDigits / 64;
            const int at = threadIdx.x * N;
            u64 sums[N], w = 0;
            unsigned counts[N], c = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                w += sums[i] = s.digit_sum[at + i];
                c += counts[i] = s.digit_count[at + i];
                s.digit_sum[at + i] = 0;
                s.digit_count[at + i] = 0;
            }
            const u64 win = wave_scan(w);
            const unsigned cin = wave_scan(c);
            find_among<N>(s, b, sums, counts, at, count + cin - c, sum + win - w, c, w, none);
        }
        __syncthreads();
        const int bin = s.found;
        const unsigned many = s.found_many;
        count = s.found_count;
        sum = s.found_sum;
        prefix |= (u64)max(bin, 0) << shift;
        if (shift == 0 || many <= kFew || bin < 0) break;
        above = shift;
        shift = max(shift - kDigit, 0);
        __syncthreads();
    }
    // the items in the last bin
    if (threadIdx.x == 0) s.few = 0;
    __syncthreads();
    items.go([&](u64 code, u64 w) {
        if ((code - low) >> shift != prefix >> shift) return;
        const int i = atomicAdd(&s.few, 1);
        if (i < kFew) s.few_code[i] = code, s.few_weight[i] = w;
    });
    __syncthreads();
    const int few = min(s.few, kFew);
    if ((int)threadIdx.x < few) {
        const u64 code = s.few_code[threadIdx.x], w = s.few_weight[threadIdx.x];
#pragma unroll 4
        for (int i = 0; i < few; ++i) {
            const bool before = s.few_code[i] < code;
            count += before ? 1 : 0;
            sum += before ? s.few_weight[i] : 0;
        }
        if (!(count > none && b.reached(count, sum)) && b.reached(count + 1, sum + w)) s.found_code = code, s.found_sum = w;
    }
    __syncthreads();
    const u64 code = s.found_code;
    weight = s.found_sum;
    __syncthreads();
    return code;
}

// ---------------------------------------------------------------- sorted lists
// The value of the lane whose number differs in one bit.  (`tid` is handed on from where the
// compiler cannot tell what it is: it would keep a mask for each step in registers from row to row.)
template <int BIT>
CNN_INLINE unsigned across(unsigned v, int tid) {
    if constexpr (BIT == 1) return moved<0xb1, 0xf>(v);                        // quad_perm 1 0 3 2
    else if constexpr (BIT == 2) return moved<0x4e, 0xf>(v);                   // quad_perm 2 3 0 1
    else if constexpr (BIT == 4) return moved<0x1b, 0xf>(moved<0x141, 0xf>(v));  // half a row's mirror, and a quad's
    else if constexpr (BIT == 8) return moved<0x128, 0xf>(v);                  // row_ror 8
    else {
        // rows (halves) of two copies exchanged: one has the even ones twice, the other the odd ones
        const auto p = BIT == 16 ? __builtin_amdgcn_permlane16_swap(v, v, false, false) : __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return tid & BIT ? p[0] : p[1];
    }
}
template <int BIT>
CNN_INLINE u64 across(u64 v, int tid) { return (u64)across<BIT>((unsigned)(v >> 32), tid) << 32 | across<BIT>((unsigned)v, tid); }

// A step of a bitonic network between lanes BIT apart; up: the lower lane gets the lower code.
template <int BIT>
CNN_INLINE u64 exchange(u64 code, int tid, bool up) {
    const u64 other = across<BIT>(code, tid);
    return (code < other) == (((tid & BIT) == 0) == up) ? code : other;
}
CNN_INLINE u64 merge_wave(u64 code, int tid, bool up) {
    code = exchange<32>(code, tid, up);
    code = exchange<16>(code, tid, up);
    code = exchange<8>(code, tid, up);
    code = exchange<4>(code, tid, up);
    code = exchange<2>(code, tid, up);
    return exchange<1>(code, tid, up);
}
// Sorts one code of each of the first `many` work-items (a power of two, 64 at least): a
// bitonic network, within waves by moves between lanes, between waves through LDS.
CNN_INLINE u64 sort_codes(u64* room, u64 code, int many) {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    auto up = [&](int k) { return (tid & k) == 0; };
    if (tid < many) {
        code = exchange<1>(code, tid, up(2));
        code = exchange<2>(code, tid, up(4));
        code = exchange<1>(code, tid, up(4));
        code = exchange<4>(code, tid, up(8));
        code = exchange<2>(code, tid, up(8));
        code = exchange<1>(code, tid, up(8));
        code = exchange<8>(code, tid, up(16));
        code = exchange<4>(code, tid, up(16));
        code = exchange<2>(code, tid, up(16));
        code = exchange<1>(code, tid, up(16));
        code = exchange<16>(code, tid, up(32));
        code = exchange<8>(code, tid, up(32));
        code = exchange<4>(code, tid, up(32));
        code = exchange<2>(code, tid, up(32));
        code = exchange<1>(code, tid, up(32));
        code = merge_wave(code, tid, up(64));
    }
#pragma unroll 1
    for (int k = 128; k <= many; k <<= 1) {
#pragma unroll 1
        for (int j = k >> 1; j >= 64; j >>= 1) {
            __syncthreads();
            if (tid < many) room[tid] = code;
            __syncthreads();
            if (tid < many) {
                const u64 other = room[tid ^ j];
                code = (code < other) == (((tid & j) == 0) == up(k)) ? code : other;
            }
        }
        if (tid < many) code = merge_wave(code, tid, up(k));
    }
    return code;
}
CNN_INLINE int power_of_two(int n) {
    int many = 64;
    while (many < n) many <<= 1;
    return many;
}
// A work-item's code of the list's n (blockDim.x at most) in order, or kAll.
CNN_INLINE u64 sorted(List& list, int n) {
    const u64 code = (int)threadIdx.x < n ? list.code[threadIdx.x] : kAll;
    __syncthreads();
    return sort_codes(list.code, code, power_of_two(n));
}

// The whole number that u of a sum is.
CNN_INLINE u64 share_of(float u, u64 sum) {
    const double r = (double)fmaxf(u, 0.0f) * (double)sum;
    const u64 t = r < 0x1p63 ? (u64)r : sum;
    return min(t, sum - 1);
}

// As find_code, among a list's n <= blockDim.x codes, which are sorted.
template <int NT>
CNN_INLINE u64 find_sorted(Shared<NT>& s, List& list, const Row& r, int n, const Border& b, u64 count, u64 sum) {
    const u64 code = sorted(list, n);
    const bool there = code != kAll;
    u64 all;
    const u64 w = there ? r.scale.weight(value_of(code)) : 0, upto = sum + group_scan(s, w, all);
    count += threadIdx.x;  // before this one
    if (there && !(threadIdx.x > 0 && b.reached(count, upto - w)) && b.reached(count + 1, upto)) s.found_code = code;
    __syncthreads();
    return s.found_code;
}

struct Drawn {
    int token;
    float prob;
};
// The rest of a row, all that it keeps being among the n <= blockDim.x codes of the list.  total: the weight
// that top-p is a share of; 0: that of the first top_k codes.
template <int NT>
CNN_INLINE Drawn draw_sorted(Shared<NT>& s, List& list, const Row& r, int n, u64 total) {
    const int tid = threadIdx.x;
    const u64 code = sorted(list, n);
    const bool there = code != kAll;
    u64 all;
    const u64 w = there ? r.scale.weight(value_of(code)) : 0, sum = group_scan(s, w, all);
    if (total == 0) {
        if (tid == (r.cut_k ? min(r.top_k, (int)blockDim.x) : (int)blockDim.x) - 1) s.found_sum = sum;
        __syncthreads();
        total = s.found_sum;
    }
    bool keep = there && (w >= r.least || tid == 0);
    if (r.cut_k) keep = keep && tid < r.top_k;
    if (r.cut_p) keep = keep && (tid == 0 || (double)(sum - w) < (double)r.top_p * (double)total);
    // the kept ones are the first ones
    const int kept = (int)group_max(s, keep ? tid + 1 : 0);
    const u64 by_number = sort_codes(list.code, keep ? code << 32 | code >> 32 : kAll, power_of_two(kept));
    const u64 v = by_number != kAll ? r.scale.weight(value_of(by_number << 32)) : 0, upto = group_scan(s, v, all);
    const u64 beyond = share_of(r.u, all);
    if (upto > beyond && upto - v <= beyond) s.found_code = by_number >> 32, s.found_sum = v;
    __syncthreads();
    return Drawn{(int)s.found_code, (float)((double)s.found_sum / (double)all)};
}

// ---------------------------------------------------------------- passes over a row
// The largest logit and its first token, as one number (0: there is none).
template <int NT, typename T>
CNN_INLINE u64 largest(Shared<NT>& s, const T* x, int64_t from, int64_t to, int V) {
    float most = -INFINITY, v[8];
    int at = 0, first = 0;
    each_eight(x, from, to, V, [&](int c, const float* l) {  // (fmaxf leaves NaN out)
        const float m = fmaxf(fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3])), fmaxf(fmaxf(l[4], l[5]), fmaxf(l[6], l[7])));
        if (m > most) most = m, at = c;
    });
    if (most > -INFINITY) {
        load_logits(x, at, to, V, v);
#pragma unroll
        for (int i = 7; i >= 0; --i) first = v[i] == most ? at + i : first;
    }
    return group_max(s, most > -INFINITY ? (u64)key_of(most + 0.0f) << 32 | (unsigned)~first : 0);
}

// Adds the tokens that are kept by code to the bins by weight; without `weigh` only their number.  Tokens
// of the last bin weigh nothing and are left out.
template <int NT, typename T>
CNN_INLINE void add_by_weight(Shared<NT>& s, const T* x, int64_t from, int64_t to, int V, const Row& r, bool weigh, u64 last) {
    if (weigh) {
        each_logit(x, from, to, V, [&](int i, float l) {
            const float v = r.scale.value(l);
            const int b = r.scale.bin(v);  // the last one for minus infinity
            if (b >= kBins - 1 || (last != kAll && code_of(v, i) > last)) return;
            atomicAdd(&s.sum[b], r.scale.weight(v));
            atomicAdd(&s.count[b], 1u);
        });
    } else if (r.scale.infinite) {
        each_logit(x, from, to, V, [&](int, float l) {
            if (l == INFINITY) atomicAdd(&s.count[0], 1u);
        });
    } else {
        each_logit(x, from, to, V, [&](int, float l) {
            const int b = r.scale.bin(l);
            if (b < kBins - 1) atomicAdd(&s.count[b], 1u);
        });
    }
}

// The weights of 8 tokens from c on, 0 for those that are not kept; returns their sum.
template <typename T>
CNN_INLINE u64 kept_weights(const T* x, int64_t c, int V, const Row& r, u64 last, u64* w) {
    float l[8];
    load_logits(x, c, V, V, l);
    u64 sum = 0;
    if (last == kAll && r.least == 0 && !r.scale.infinite) {  // minus infinity and NaN weigh nothing
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += w[i] = r.scale.weight(l[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = r.scale.value(l[i]);
            const u64 code = code_of(v, (int)c + i);
            w[i] = 0;
            if (v > -INFINITY && code <= last) {
                w[i] = r.scale.weight(v);
                if (!r.keeps(code, w[i], last)) w[i] = 0;
            }
            sum += w[i];
        }
    }
    return sum;
}
// The weight of a tile's kept tokens, in every lane of the wave that calls it.
template <typename T>
CNN_INLINE u64 tile_sum(const T* x, int64_t from, int64_t to, int V, const Row& r, u64 last) {
    u64 sum = 0, w[8];
    for (int64_t c = from + (threadIdx.x & 63) * 8; c < to; c += 512) sum += kept_weights(x, c, V, r, last, w);
    return wave_sum(sum);
}
// The token of a tile at which the sum, `before` in front of the tile, exceeds `beyond`, by one wave.
template <int NT, typename T>
CNN_INLINE void draw_in_tile(Shared<NT>& s, const T* x, int64_t from, int64_t to, int V, const Row& r, u64 last, u64 before, u64 beyond) {
    const int lane = threadIdx.x & 63;
#pragma unroll 1
    for (int64_t c = from; c < to; c += 512) {
        u64 w[8];
        const int64_t at = c + lane * 8;
        const u64 mine = at < to ? kept_weights(x, at, V, r, last, w) : 0, upto = before + wave_scan(mine);
        if (upto > beyond && upto - mine <= beyond) {
            u64 sum = upto - mine;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (sum <= beyond && sum + w[i] > beyond) s.found_code = (u64)(at + i), s.found_sum = w[i];
                sum += w[i];
            }
        }
        before = last_lane(upto);
        if (before > beyond) break;
    }
}

// put(code) for the tokens kept by code of the bins first..end, between two places of the row.
template <typename T, typename F>
CNN_INLINE void each_in_bins(const T* x, int64_t from, int64_t to, int V, const Row& r, int first, int end, u64 last, F&& put) {
    auto in = [&](int i, float v) {
        const int b = r.scale.bin(v);
        if (b < first || b > end) return;
        const u64 code = code_of(v + 0.0f, i);
        if (code <= last) put(code);
    };
    if (r.scale.infinite) each_logit(x, from, to, V, [&](int i, float l) { in(i, r.scale.value(l)); });
    else each_logit(x, from, to, V, in);
}
// The weights of the list's codes.
CNN_INLINE void weigh_list(List& list, const Row& r, int n) {
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const u64 code = list.code[i];
        list.weight[i] = r.scale.weight(value_of(code));
    }
    __syncthreads();
}

// ---------------------------------------------------------------- kernels
CNN_INLINE u64 best_of(const Split& sp, int row) {
    u64 best = 0;
    for (int c = threadIdx.x & 63; c < sp.chunks; c += 64) best = max(best, sp.best[(size_t)row * sp.chunks + c]);
    return wave_max(best);
}
template <int NT>
CNN_INLINE void load_bins(Shared<NT>& s, const Split& sp, int row, int n) {
    for (int i = threadIdx.x; i < kBins; i += blockDim.x) {
        s.sum[i] = i < n ? sp.sum[(size_t)row * kBins + i] : 0;
        s.count[i] = i < n ? sp.count[(size_t)row * kBins + i] : 0;
    }
    __syncthreads();
}
template <int NT>
CNN_INLINE u64 sum_of_bins(Shared<NT>& s) {
    u64 mine = 0;
    for (int i = threadIdx.x; i < kBins; i += blockDim.x) mine += s.sum[i];
    return group_sum(s, mine);
}
// Which tokens go to the list: all that may be kept (bins from 0), those of the border's bin, or none.
struct Choice {
    bool all, listed;
    CNN_INLINE explicit Choice(const Place& at) {
        all = at.count + at.many <= kList;
        listed = all || at.many <= (unsigned)kList;
    }
};

// What a workgroup does with a row: all of it; the cuts, of which the first has its bins and its list in the
// workspace; the draw, whose tiles are there.
enum Mode { WHOLE, CUTS, LAST };

template <typename T, int MODE, int NT>
__global__ void __launch_bounds__(NT) sample_rows(Args a) {
    __shared__ Shared<NT> s;
    __shared__ List list;
    const Sample& p = a.p;
    const Split& sp = a.split;
    const int V = p.V, tid = threadIdx.x, wave = tid >> 6, waves = blockDim.x >> 6;
    const int tiles = (int)(((int64_t)V + a.each - 1) / a.each);
    for (int i = tid; i < kDigits; i += blockDim.x) s.digit_sum[i] = 0, s.digit_count[i] = 0;
    for (int row = blockIdx.x; row < p.N; row += gridDim.x) {
        const T* x = (const T*)p.logits + (size_t)row * V;
        const Parameters q(p, row);
        const u64 best = MODE == WHOLE ? largest(s, x, 0, V, V) : best_of(sp, row);
        const Row r(a, q, best);
        auto done = [&](int token, float prob) {
            if (tid != 0) return;
            p.token[row] = token;
            if (p.prob) p.prob[row] = prob;
            if (MODE == CUTS) sp.pending[row] = 0;
        };
        if (r.token != -2) {
            done(r.token, r.prob);
            continue;
        }
        u64 last = kAll;        // the code of the last token kept
        bool in_list = false;   // the list holds all that are kept
        bool filled = MODE != WHOLE;  // the first bins wait in the workspace
        if (MODE == LAST && sp.pending) {
            if (!sp.pending[row]) continue;
            last = sp.last[row];
        }
        if (MODE == WHOLE && V <= 256) {
            const float v = tid < V ? r.scale.value(to_f32(x[tid])) : -INFINITY;
            if (tid < V) list.code[tid] = v > -INFINITY ? code_of(v, tid) : kAll;
            const Drawn d = draw_sorted(s, list, r, V, 0);
            done(d.token, d.prob);
            continue;
        }
#pragma unroll 1
        for (int kind = MODE == LAST ? DRAW : COUNT; kind <= DRAW; ++kind) {
            if ((kind == COUNT && !r.cut_k) || (kind == SHARE && !r.cut_p)) continue;
            if (MODE == CUTS && kind == DRAW && !in_list) {
                if (tid == 0) sp.last[row] = last, sp.pending[row] = 1;
                break;
            }
            Items<T> items{x, V, r, list, in_list ? s.listed : -1, kind, 0, last};
            u64 count = 0, sum = 0, total = 0;
            if (in_list) {
                u64 mine = 0;
                items.go([&](u64, u64 w) { mine += w; });
                total = group_sum(s, mine);
            } else {
                if (filled) {
                    load_bins(s, sp, row, kind == DRAW ? tiles : kBins);
                } else {
                    clear_bins(s);
                    if (kind != DRAW) {
                        add_by_weight(s, x, 0, V, V, r, kind == SHARE, last);
                    } else {
                        for (int t = wave; t < tiles; t += waves) {
                            const int64_t from = (int64_t)t * a.each;
                            const u64 w = tile_sum(x, from, min(from + a.each, (int64_t)V), V, r, last);
                            if ((tid & 63) == 0) s.sum[t] = w, s.count[t] = 1;
                        }
                    }
                    __syncthreads();
                }
                if (kind != COUNT) total = sum_of_bins(s);
            }
            const Border b{kind, (u64)r.top_k, (double)r.top_p * (double)total, kind == DRAW ? share_of(r.u, total) : 0};
            if (!in_list) {
                const Place at = find_bin(s, b);
                if (kind == DRAW) {
                    const int64_t from = (int64_t)at.bin * a.each;
                    if (wave == 0) draw_in_tile(s, x, from, min(from + a.each, (int64_t)V), V, r, last, at.sum, b.beyond);
                    __syncthreads();
                    done((int)s.found_code, (float)((double)s.found_sum / (double)total));
                    break;
                }
                const bool was_filled = filled;
                filled = false;
                if (at.bin < 0) continue;  // fewer tokens weigh anything than top-k keeps
                const Choice choice(at);
                if (choice.listed) {
                    if (MODE == CUTS && was_filled) {
                        const int n = sp.listed[row];
                        for (int i = tid; i < n; i += blockDim.x) list.code[i] = sp.list[(size_t)row * kList + i];
                        if (tid == 0) s.listed = n;
                    } else {
                        if (tid == 0) s.listed = 0;
                        __syncthreads();
                        each_in_bins(x, 0, V, V, r, choice.all ? 0 : at.bin, at.bin, last, [&](u64 code) {
                            const int i = atomicAdd(&s.listed, 1);
                            if (i < kList) list.code[i] = code;
                        });
                    }
                    __syncthreads();
                    items.listed = s.listed;
                }
                if (!choice.all) count = at.count, sum = at.sum;
                if (choice.listed && items.listed <= (int)blockDim.x) {
                    if (choice.all) {
                        const Drawn d = draw_sorted(s, list, r, items.listed, total);
                        done(d.token, d.prob);
                        break;
                    }
                    last = find_sorted(s, list, r, items.listed, b, count, sum);
                    continue;
                }
                if (choice.listed) weigh_list(list, r, items.listed);
                items.bin = at.bin;
                in_list = choice.all;
            }
            u64 weight;
            const u64 code = find_code(s, items, b, count, sum, weight);
            if (kind != DRAW) last = code;
            else done((int)code, (float)((double)weight / (double)total));
        }
        __syncthreads();  // what was found and listed is the next row's
    }
}

constexpr int kChunkThreads = 512, kTileThreads = 256;

// A chunk's largest logit; the row's bins and its list are cleared on the way.
template <typename T>
__global__ void __launch_bounds__(kChunkThreads) sample_best(Args a) {
    __shared__ Shared<kChunkThreads> s;
    const Split& sp = a.split;
    const int row = blockIdx.x / (unsigned)sp.chunks, c = blockIdx.x % (unsigned)sp.chunks, V = a.p.V;
    const int64_t from = (int64_t)c * sp.chunk, to = min(from + sp.chunk, (int64_t)V);
    for (int i = c * kChunkThreads + threadIdx.x; i < kBins; i += sp.chunks * kChunkThreads)
        sp.sum[(size_t)row * kBins + i] = 0, sp.count[(size_t)row * kBins + i] = 0;
    const u64 best = largest(s, (const T*)a.p.logits + (size_t)row * V, from, to, V);
    if (threadIdx.x == 0) {
        sp.best[(size_t)row * sp.chunks + c] = best;
        if (c == 0) sp.listed[row] = 0;
    }
}

// A chunk's part of the bins that the row's first cut is found by.
template <typename T>
__global__ void __launch_bounds__(kChunkThreads) sample_bins(Args a) {
    __shared__ Shared<kChunkThreads> s;
    const Split& sp = a.split;
    const int row = blockIdx.x / (unsigned)sp.chunks, c = blockIdx.x % (unsigned)sp.chunks, V = a.p.V;
    const int64_t from = (int64_t)c * sp.chunk, to = min(from + sp.chunk, (int64_t)V);
    const Row r(a, Parameters(a.p, row), best_of(sp, row));
    if (r.token != -2 || !(r.cut_k || r.cut_p)) return;
    clear_bins(s);
    add_by_weight(s, (const T*)a.p.logits + (size_t)row * V, from, to, V, r, !r.cut_k, kAll);
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kChunkThreads) {
        if (s.sum[i]) atomicAdd(&sp.sum[(size_t)row * kBins + i], s.sum[i]);
        if (s.count[i]) atomicAdd(&sp.count[(size_t)row * kBins + i], s.count[i]);
    }
}

// A chunk's tokens for the list of the row's first cut.  (Their order in it is that in which they come: nothing
// depends on it.)
template <typename T>
__global__ void __launch_bounds__(kChunkThreads) sample_gather(Args a) {
    __shared__ Shared<kChunkThreads> s;
    __shared__ u64 codes[kList];
    __shared__ int place;
    const Split& sp = a.split;
    const int row = blockIdx.x / (unsigned)sp.chunks, c = blockIdx.x % (unsigned)sp.chunks, V = a.p.V;
    const int64_t from = (int64_t)c * sp.chunk, to = min(from + sp.chunk, (int64_t)V);
    const Row r(a, Parameters(a.p, row), best_of(sp, row));
    if (r.token != -2 || !(r.cut_k || r.cut_p)) return;
    load_bins(s, sp, row, kBins);
    const int kind = r.cut_k ? COUNT : SHARE;
    const u64 total = kind == SHARE ? sum_of_bins(s) : 0;
    const Place at = find_bin(s, Border{kind, (u64)r.top_k, (double)r.top_p * (double)total, 0});
    if (at.bin < 0) return;
    const Choice choice(at);
    if (!choice.listed) return;
    if (threadIdx.x == 0) s.listed = 0;
    __syncthreads();
    each_in_bins((const T*)a.p.logits + (size_t)row * V, from, to, V, r, choice.all ? 0 : at.bin, at.bin, kAll, [&](u64 code) {
        const int i = atomicAdd(&s.listed, 1);
        if (i < kList) codes[i] = code;
    });
    __syncthreads();
    const int n = min(s.listed, kList);
    if (threadIdx.x == 0 && n > 0) place = atomicAdd(&sp.listed[row], n);
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kChunkThreads)
        if (place + i < kList) sp.list[(size_t)row * kList + place + i] = codes[i];
}

// The tiles of a row whose draw is pending, one a wave.
template <typename T>
__global__ void __launch_bounds__(kTileThreads) sample_tiles(Args a, int groups) {
    const Split& sp = a.split;
    const int row = blockIdx.x / (unsigned)groups, V = a.p.V;
    const int64_t tile = (int64_t)(blockIdx.x % (unsigned)groups) * (kTileThreads / 64) + (threadIdx.x >> 6), from = tile * a.each;
    if (from >= V || (sp.pending && !sp.pending[row])) return;
    const Row r(a, Parameters(a.p, row), best_of(sp, row));
    if (r.token != -2) return;
    const u64 w = tile_sum((const T*)a.p.logits + (size_t)row * V, from, min(from + a.each, (int64_t)V), V, r, sp.pending ? sp.last[row] : kAll);
    if ((threadIdx.x & 63) == 0) sp.sum[(size_t)row * kBins + tile] = w, sp.count[(size_t)row * kBins + tile] = 1;
}

// The bits that a weight is held to: V of the largest still fit 64.
int weight_bits(int V) {
    const int log2 = V > 1 ? 32 - __builtin_clz((unsigned)V - 1) : 0;
    return std::min(51, 63 - log2);
}

// A tile: as many tokens as a wave loads at a time, or more where that were more than kBins tiles.
int tile_tokens(int V) { return 512 * (int)ceil_div64(V, 512 * kBins); }

// Rows are split where there are too few for all compute units, and long: six launches instead of one, or three where
// there is no top-k or top-p.  Both ways took the same time, in fp32 with top-k and top-p, at
// 1 x 32768 (29 us) and 64 x 50021 (54), without at 1 x 16384 (12.5) and 128 x 32768 (20.5); at 1 x 131072
// it is 71 and 30 us, and 47 and 13.
int chunks_of(int N, int V, bool cuts) {
    if (N > 128 || V < (cuts ? 36000 + 300 * N : 16000 + 150 * N)) return 0;
    const int each = tile_tokens(V);
    const int64_t most = std::min<int64_t>(512 / N, V / 4096);
    return most < 2 ? 0 : (int)ceil_div64(V, ceil_div64(ceil_div64(V, most), each) * each);
}

// The workspace of a call that splits rows (base: or NULL, to know its size).
size_t lay_out(Split& sp, int N, int V, bool cuts, char* base) {
    const int each = tile_tokens(V);
    sp.chunks = chunks_of(N, V, cuts);
    if (sp.chunks == 0) return 0;
    sp.chunk = (int)(ceil_div64(ceil_div64(V, sp.chunks), each) * each);
    size_t at = 0;
    auto take = [&](auto*& p, size_t n) {
        p = (std::remove_reference_t<decltype(p)>)(base + at);
        at += (n * sizeof(*p) + 7) / 8 * 8;
    };
    take(sp.sum, (size_t)N * kBins);
    take(sp.best, (size_t)N * sp.chunks);
    take(sp.last, N);
    take(sp.list, (size_t)N * kList);
    take(sp.listed, N);
    take(sp.count, (size_t)N * kBins);
    take(sp.pending, N);
    return at;
}

template <typename T, int NT>
void run_rows(const Args& a, const dim3& rows, hipStream_t st) {
    enqueue(sample_rows<T, WHOLE, NT>, rows, dim3(NT), 0, st, a);
}
template <typename T>
void run(const Args& a, bool cuts, hipStream_t st) {
    const dim3 rows((unsigned)std::min(a.p.N, 1 << 20));
    if (a.split.chunks == 0) {
        // A workgroup's barriers cost more the larger it is, its passes less: 128 rows of 1000, 4096, 8000 with
        // cuts took 17.6, 22.8, 30.5 us with 256 work-items and 16.1, 19.3, 24.0 with 512, one of 1000 11.7 and
        // 12.1; 128 of 32768 46.9 with 512 and 42.0 with 1024, without cuts 20.5 and 20.9, of 50021 28.7 and 26.7.
        if (a.p.V <= 1024) run_rows<T, 256>(a, rows, st);
        else if (a.p.V <= (cuts ? 20000 : 40000)) run_rows<T, 512>(a, rows, st);
        else run_rows<T, 1024>(a, rows, st);
        return;
    }
    const dim3 parts((unsigned)(a.p.N * a.split.chunks)), threads(kChunkThreads);
    enqueue(sample_best<T>, parts, threads, 0, st, a);
    if (a.split.pending) {
        enqueue(sample_bins<T>, parts, threads, 0, st, a);
        enqueue(sample_gather<T>, parts, threads, 0, st, a);
        enqueue(sample_rows<T, CUTS, 512>, rows, dim3(512), 0, st, a);
    }
    const int groups = ceil_div(ceil_div(a.p.V, a.each), kTileThreads / 64);
    enqueue(sample_tiles<T>, dim3((unsigned)(a.p.N * groups)), dim3(kTileThreads), 0, st, a, groups);
    enqueue(sample_rows<T, LAST, 256>, rows, dim3(256), 0, st, a);
}

}  // namespace

size_t sample_workspace(int type, int N, int V) {
    Split sp{};
    return std::max(lay_out(sp, N, V, false, nullptr), lay_out(sp, N, V, true, nullptr));
}

int launch_sample(const Sample& p, void* ws, hipStream_t st) {
    if (p.N == 0) return CNN_OK;
    Args a{p, weight_bits(p.V), tile_tokens(p.V), {}};
    const bool cuts = p.top_k || p.top_p;
    lay_out(a.split, p.N, p.V, cuts, (char*)ws);
    if (!cuts) a.split.pending = nullptr;
    if (p.type == CNN_F32) run<float>(a, cuts, st);
    else if (p.type == CNN_BF16) run<bf16_t>(a, cuts, st);
    else run<f16_t>(a, cuts, st);
    return check_launch("sample");
}

}  // namespace cnn
