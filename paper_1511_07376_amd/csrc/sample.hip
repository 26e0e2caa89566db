// A token for each row of logits: temperature, top-k, top-p, min-p, then the token that a
// random number of the caller's falls on.
//
// Which token that is, and where top-p ends, is a matter of sums next to a border, so
// weights exp((l - max l) / T) are taken as whole numbers of 2^-S of the largest (S = 51, less
// where 2^S times V would pass 64 bits) from an exponential in 64-bit floats.  Their sums
// are exact, whatever the order: additions can be atomic, split, and done twice with
// the same result.
//
// Nothing is sorted.  The tokens' order (falling logit, rising number) is a code of 64 bits
// for each, and the last token that a rule keeps is the one at which a count (top-k) or a
// sum (top-p) is reached: it is found by histograms, first over bins of equal width in log2 of
// the weight, then over the digits of the codes of the tokens in the bin where the
// border lies.  The draw is the same search over the tokens' numbers, whose first bins are
// tiles of the row.  Once all that a row keeps fits a list in LDS, the rest is done there.
//
// One workgroup does a row, or, where there are few long rows, several do what passes over all
// of it: the largest logit, the first histogram, the tiles' sums.
#include "f8.h"

#include <algorithm>

namespace cnn {
namespace {

typedef unsigned long long u64;

constexpr int kBins = 2048;
constexpr int kDigit = 11;              // bits of a digit: kBins values
constexpr float kBinsPerOctave = 38.0f;  // the last bin begins at 2^-53.8, which is no whole number's weight
constexpr int kList = 4096;             // tokens that are worked on in LDS
constexpr int kMostWaves = 16;
constexpr u64 kAll = ~0ull;

#define CNN_INLINE __device__ inline __attribute__((always_inline))

// What a row shares between the kernels of a call that splits rows.
struct Split {
    u64* best;      // [N][chunks] largest logit and its first token, of a chunk
    u64* last;      // [N] code of the last token kept
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
    // Not falling as the logit falls, in the same way wherever it is called.  (Halves: the
    // difference of the largest and the least float is more than a float.)
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

// A row's parameters, and what follows from them and its largest logit.
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
    CNN_INLINE Row(const Args& a, int row, u64 best) {
        const Sample& p = a.p;
        const float temperature = p.temperature ? p.temperature[row] : 1.0f, min_p = p.min_p ? p.min_p[row] : 0.0f;
        u = p.u[row];
        top_p = p.top_p ? p.top_p[row] : 1.0f;
        top_k = p.top_k ? p.top_k[row] : 0;
        first = (int)~(unsigned)best;
        token = -2;
        prob = 1.0f;
        const bool fine = temperature >= 0.0f && temperature < INFINITY && u == u && top_p == top_p && min_p == min_p;
        if (best == 0 || !fine) token = -1, prob = 0.0f;
        else if (temperature == 0.0f || top_k == 1 || top_p <= 0.0f || min_p > 1.0f) token = first;
        const unsigned key = (unsigned)(best >> 32);
        const float most = __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key);
        scale.infinite = most == INFINITY;
        scale.top = scale.infinite ? 0.0f : most;
        scale.per = 1.4426950408889634 / (double)temperature;
        scale.bins = (float)fmin(2.0 * scale.per * (double)kBinsPerOctave, 3e38);
        scale.bits = a.bits;
        first_code = code_of(scale.top, first);
        cut_k = top_k > 0 && top_k < p.V;
        cut_p = top_p < 1.0f;
        least = min_p > 0.0f ? (u64)__builtin_ceil((double)fminf(min_p, 1.0f) * (double)(1ull << a.bits)) : 0;
    }
    CNN_INLINE bool keeps(u64 code, u64 w, u64 last) const { return code <= last && (w >= least || code == first_code); }
};

// f(token, logit) for the tokens from `from` to `to` of a row of V, 8 neighbours a work-item (`from` is a
// multiple of 8).
template <typename T, typename F>
CNN_INLINE void each_logit(const T* row, int64_t from, int64_t to, int V, F&& f) {
    for (int64_t c = from + threadIdx.x * 8; c < to; c += (int64_t)blockDim.x * 8) {
        float v[8];
        load_values8(row, (int)c, V, v);
        const int n = (int)min(to - c, (int64_t)8);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) f((int)c + i, v[i]);
    }
}

// ---------------------------------------------------------------- searches
struct Shared {
    u64 sum[kBins];
    unsigned count[kBins];
    u64 wave_sum[kMostWaves];
    unsigned wave_count[kMostWaves];
    u64 low, high;  // of codes
    u64 found_sum, found_code;
    unsigned found_count, found_many;
    int found;
    int listed;
};
struct List {
    u64 weight[kList];
    u64 code[kList];
};

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

CNN_INLINE void clear_bins(Shared& s) {
    for (int i = threadIdx.x; i < kBins; i += blockDim.x) s.sum[i] = 0, s.count[i] = 0;
    __syncthreads();
}

CNN_INLINE u64 shuffle_up(u64 v, int off) {
    const unsigned lo = (unsigned)__shfl_up((int)(unsigned)v, off), hi = (unsigned)__shfl_up((int)(unsigned)(v >> 32), off);
    return (u64)hi << 32 | lo;
}
CNN_INLINE u64 shuffle_xor(u64 v, int off) {
    const unsigned lo = (unsigned)__shfl_xor((int)(unsigned)v, off), hi = (unsigned)__shfl_xor((int)(unsigned)(v >> 32), off);
    return (u64)hi << 32 | lo;
}
CNN_INLINE u64 wave_sum(u64 v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += shuffle_xor(v, off);
    return v;
}

// The sum over the workgroup, in every work-item.
CNN_INLINE u64 group_sum(Shared& s, u64 v) {
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.wave_sum[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
    for (unsigned w = 0; w < blockDim.x >> 6; ++w) v += s.wave_sum[w];
    __syncthreads();
    return v;
}

// The bin in which the border lies, what stands before the bins being (count0, sum0).
// The bins are complete (a barrier behind them).
CNN_INLINE Place find_bin(Shared& s, const Border& b, u64 count0, u64 sum0) {
    const int each = kBins / (int)blockDim.x, at = threadIdx.x * each, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    u64 w = 0;
    unsigned c = 0;
    for (int i = 0; i < each; ++i) w += s.sum[at + i], c += s.count[at + i];
    u64 win = w;
    unsigned cin = c;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const u64 uw = shuffle_up(win, off);
        const unsigned uc = (unsigned)__shfl_up((int)cin, off);
        if (lane >= off) win += uw, cin += uc;
    }
    if (threadIdx.x == 0) s.found = -1;
    if (lane == 63) s.wave_sum[wave] = win, s.wave_count[wave] = cin;
    __syncthreads();
    u64 sum = sum0 + win - w, count = count0 + cin - c;
    for (int v = 0; v < wave; ++v) sum += s.wave_sum[v], count += s.wave_count[v];
    // Before this work-item's bins it is not reached, behind them it is: in one work-item only.  (A
    // border that nothing reaches is at the first token.)
    if (c > 0 && !(count > count0 && b.reached(count, sum)) && b.reached(count + c, sum + w)) {
        for (int i = 0; i < each; ++i) {
            const u64 bw = s.sum[at + i];
            const unsigned bc = s.count[at + i];
            if (bc > 0 && b.reached(count + bc, sum + bw)) {
                s.found = at + i;
                s.found_sum = sum;
                s.found_count = (unsigned)count;
                s.found_many = bc;
                break;
            }
            sum += bw, count += bc;
        }
    }
    __syncthreads();
    const Place p{s.found, s.found_count, s.found_sum, s.found_many};
    __syncthreads();
    return p;
}

// The tokens that a search is among: those of the list, or those of the row that fall into a first bin
// (of weights, or a tile).  Of them the ones that are kept.
template <typename T>
struct Items {
    const T* x;
    int V, each;
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
            // as rare as it is slow: more tokens in a bin than the list holds
            const int64_t from = kind == DRAW ? (int64_t)bin * each : 0, to = kind == DRAW ? min(from + each, (int64_t)V) : V;
#pragma unroll 1
            for (int64_t i = from + threadIdx.x; i < to; i += blockDim.x) {
                const float v = r.scale.value(to_f32(x[i]));
                if (v == -INFINITY || (kind != DRAW && r.scale.bin(v) != bin)) continue;
                const u64 code = code_of(v, (int)i), w = kind == COUNT ? 0 : r.scale.weight(v);
                if (kind != DRAW ? code <= last : r.keeps(code, w, last)) f(kind == DRAW ? (u64)i : code, w);
            }
        }
    }
};

// The first code, of the items' in rising order, at which the border is reached: there is one.  Before
// all of the items: (count, sum).  `weight`: the found one's.
template <typename T>
CNN_INLINE u64 find_code(Shared& s, const Items<T>& items, const Border& b, u64 count, u64 sum, u64& weight) {
    if (threadIdx.x == 0) s.low = kAll, s.high = 0;
    __syncthreads();
    u64 low = kAll, high = 0;
    items.go([&](u64 code, u64) { low = min(low, code), high = max(high, code); });
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) low = min(low, shuffle_xor(low, off)), high = max(high, shuffle_xor(high, off));
    if ((threadIdx.x & 63) == 0) atomicMin(&s.low, low), atomicMax(&s.high, high);
    __syncthreads();
    const u64 base = s.low, range = s.high - s.low;
    int shift = range == 0 ? 0 : max(64 - __builtin_clzll(range) - kDigit, 0);
    u64 prefix = 0;  // of what is behind base, its digits so far; lower ones 0
    int above = 64;  // bits from here on are the prefix's
#pragma unroll 1
    for (;;) {
        clear_bins(s);
        items.go([&](u64 code, u64 w) {
            const u64 rel = code - base;
            if (above < 64 && rel >> above != prefix >> above) return;
            const int digit = (int)(rel >> shift) & (kBins - 1);
            atomicAdd(&s.sum[digit], w);
            atomicAdd(&s.count[digit], 1u);
        });
        __syncthreads();
        const Place at = find_bin(s, b, count, sum);
        prefix |= (u64)max(at.bin, 0) << shift;
        count = at.count;
        sum = at.sum;
        if (shift == 0 || at.many == 1 || at.bin < 0) break;
        above = shift;
        shift = max(shift - kDigit, 0);
    }
    // the one item in the last bin
    items.go([&](u64 code, u64 w) {
        if ((code - base) >> shift == prefix >> shift) s.found_code = code, s.found_sum = w;
    });
    __syncthreads();
    const u64 code = s.found_code;
    weight = s.found_sum;
    __syncthreads();
    return code;
}

// The whole number that u of a sum is.
CNN_INLINE u64 share_of(float u, u64 sum) {
    const double r = (double)fmaxf(u, 0.0f) * (double)sum;
    const u64 t = r < 0x1p63 ? (u64)r : sum;
    return min(t, sum - 1);
}

// ---------------------------------------------------------------- passes over a row
// The largest logit and its first token, as one number (0: there is none).
template <typename T>
CNN_INLINE u64 largest(Shared& s, const T* x, int64_t from, int64_t to, int V) {
    u64 best = 0;
    each_logit(x, from, to, V, [&](int i, float l) {
        if (l > -INFINITY) best = max(best, (u64)key_of(l + 0.0f) << 32 | (unsigned)~i);
    });
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) best = max(best, shuffle_xor(best, off));
    if ((threadIdx.x & 63) == 0) s.wave_sum[threadIdx.x >> 6] = best;
    __syncthreads();
    best = 0;
    for (unsigned w = 0; w < blockDim.x >> 6; ++w) best = max(best, s.wave_sum[w]);
    __syncthreads();
    return best;
}

// Adds the tokens kept by number `last` to the bins by weight.  Tokens of the last bin weigh nothing
// and are left out.
template <typename T>
CNN_INLINE void add_by_weight(Shared& s, const T* x, int64_t from, int64_t to, int V, const Row& r, bool weigh, u64 last) {
    if (weigh) {
        each_logit(x, from, to, V, [&](int i, float l) {
            const float v = r.scale.value(l);
            if (v == -INFINITY) return;
            const int b = r.scale.bin(v);
            if (b == kBins - 1 || code_of(v, i) > last) return;
            atomicAdd(&s.sum[b], r.scale.weight(v));
            atomicAdd(&s.count[b], 1u);
        });
    } else {
        each_logit(x, from, to, V, [&](int i, float l) {
            const float v = r.scale.value(l);
            if (v == -INFINITY) return;
            const int b = r.scale.bin(v);
            if (b != kBins - 1) atomicAdd(&s.count[b], 1u);
        });
    }
}

// The weight of a tile's kept tokens, in every lane of the wave that calls it.
template <typename T>
CNN_INLINE u64 tile_sum(const T* x, int64_t from, int64_t to, int V, const Row& r, u64 last) {
    u64 sum = 0;
    for (int64_t c = from + (threadIdx.x & 63) * 8; c < to; c += 512) {
        float l[8];
        load_values8(x, (int)c, V, l);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = c < V - i ? r.scale.value(l[i]) : -INFINITY;
            const u64 code = code_of(v, (int)c + i);
            if (v > -INFINITY && code <= last) {
                const u64 w = r.scale.weight(v);
                sum += r.keeps(code, w, last) ? w : 0;
            }
        }
    }
    return wave_sum(sum);
}

// The row's tokens of the first bins from..to (tiles in a draw), in the list.
template <typename T>
CNN_INLINE void gather(Shared& s, List& list, const T* x, int V, int each, const Row& r, int kind, int from, int to, u64 last) {
    if (threadIdx.x == 0) s.listed = 0;
    __syncthreads();
    const int64_t begin = kind == DRAW ? (int64_t)from * each : 0, end = kind == DRAW ? min((int64_t)to * each + each, (int64_t)V) : V;
    each_logit(x, begin, end, V, [&](int i, float l) {
        const float v = r.scale.value(l);
        if (v == -INFINITY) return;
        const u64 code = code_of(v, i);
        if (code > last) return;
        if (kind != DRAW) {
            const int b = r.scale.bin(v);
            if (b < from || b > to) return;
        }
        const int at = atomicAdd(&s.listed, 1);
        if (at < kList) {
            list.code[at] = code;
            list.weight[at] = r.scale.weight(v);
        }
    });
    __syncthreads();
}

// ---------------------------------------------------------------- kernels
// What a workgroup does with a row: all of it; the cuts, of which the first has its bins in the
// workspace; the draw, whose tiles are there.
enum Mode { WHOLE, CUTS, LAST };

template <typename T, int MODE>
__global__ void __launch_bounds__(1024) sample_rows(Args a) {
    __shared__ Shared s;
    __shared__ List list;
    const Sample& p = a.p;
    const Split& sp = a.split;
    const int V = p.V, tid = threadIdx.x, wave = tid >> 6, waves = blockDim.x >> 6;
    const int tiles = (int)(((int64_t)V + a.each - 1) / a.each);
    for (int row = blockIdx.x; row < p.N; row += gridDim.x) {
        __syncthreads();
        const T* x = (const T*)p.logits + (size_t)row * V;
        u64 best = 0;
        if (MODE == WHOLE) {
            best = largest(s, x, 0, V, V);
        } else {
            for (int c = 0; c < sp.chunks; ++c) best = max(best, sp.best[(size_t)row * sp.chunks + c]);
        }
        const Row r(a, row, best);
        if (r.token != -2) {
            if (tid == 0) {
                p.token[row] = r.token;
                if (p.prob) p.prob[row] = r.prob;
                if (MODE == CUTS) sp.pending[row] = 0;
            }
            continue;
        }
        u64 last = kAll;        // the code of the last token kept
        bool in_list = false;   // the list holds all that are kept
        bool filled = MODE == CUTS;  // the first bins wait in the workspace
        if (MODE == LAST && sp.pending) {
            if (!sp.pending[row]) continue;
            last = sp.last[row];
        }
#pragma unroll 1
        for (int kind = MODE == LAST ? DRAW : COUNT; kind <= DRAW; ++kind) {
            if ((kind == COUNT && !r.cut_k) || (kind == SHARE && !r.cut_p)) continue;
            if (MODE == CUTS && kind == DRAW && !in_list) {
                if (tid == 0) sp.last[row] = last, sp.pending[row] = 1;
                break;
            }
            Items<T> items{x, V, a.each, r, list, in_list ? s.listed : -1, kind, 0, last};
            u64 count = 0, sum = 0, total = 0;
            if (in_list) {
                u64 mine = 0;
                if (kind != COUNT) items.go([&](u64, u64 w) { mine += w; });
                total = group_sum(s, mine);
            } else {
                if (filled || (MODE == LAST && kind == DRAW)) {
                    const int n = kind == DRAW ? tiles : kBins;
                    for (int i = tid; i < kBins; i += blockDim.x) {
                        s.sum[i] = i < n ? sp.sum[(size_t)row * kBins + i] : 0;
                        s.count[i] = i < n ? sp.count[(size_t)row * kBins + i] : 0;
                    }
                    filled = false;
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
                }
                __syncthreads();
                if (kind != COUNT) {
                    u64 mine = 0;
                    for (int i = tid; i < kBins; i += blockDim.x) mine += s.sum[i];
                    total = group_sum(s, mine);
                }
            }
            const Border b{kind, (u64)r.top_k, (double)r.top_p * (double)total, kind == DRAW ? share_of(r.u, total) : 0};
            if (!in_list) {
                const Place at = find_bin(s, b, 0, 0);
                if (at.bin < 0) continue;  // fewer tokens weigh anything than top-k keeps
                const bool all = kind != DRAW && at.count + at.many <= kList;
                if (!all) count = at.count, sum = at.sum;
                if (all || (kind == DRAW ? a.each : (int)min(at.many, (unsigned)kList + 1)) <= kList) {
                    gather(s, list, x, V, a.each, r, kind, all ? 0 : at.bin, at.bin, last);
                    items.listed = s.listed;
                }
                items.bin = at.bin;
                in_list = all;
            }
            u64 weight;
            const u64 code = find_code(s, items, b, count, sum, weight);
            if (kind != DRAW) {
                last = code;
            } else if (tid == 0) {
                p.token[row] = (int)code;
                if (p.prob) p.prob[row] = (float)((double)weight / (double)total);
                if (MODE == CUTS) sp.pending[row] = 0;
            }
        }
    }
}

// The bits that a weight is held to: V of the largest still fit 64.
int weight_bits(int V) {
    const int log2 = V > 1 ? 32 - __builtin_clz((unsigned)V - 1) : 0;
    return std::min(51, 63 - log2);
}

// A tile: as many tokens as a wave loads at a time, or more where that were more than kBins tiles.
int tile_tokens(int V) { return 512 * (int)ceil_div64(V, 512 * kBins); }

template <typename T>
void run(const Args& a, hipStream_t st) {
    const dim3 grid((unsigned)std::min(a.p.N, 1 << 20)), block(a.p.V <= 4096 ? 256 : 1024);
    enqueue(sample_rows<T, WHOLE>, grid, block, 0, st, a);
}

}  // namespace

size_t sample_workspace(int type, int N, int V) { return 0; }

int launch_sample(const Sample& p, void* ws, hipStream_t st) {
    if (p.N == 0) return CNN_OK;
    Args a{p, weight_bits(p.V), tile_tokens(p.V), {}};
    if (p.type == CNN_F32) run<float>(a, st);
    else if (p.type == CNN_BF16) run<bf16_t>(a, st);
    else run<f16_t>(a, st);
    return check_launch("sample");
}

}  // namespace cnn
