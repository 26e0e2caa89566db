// The router of a mixture of experts, and the sum of the experts' outputs.
//
// Route.  A token's choices are its k largest logits, ties to the lower
// expert; a choice's weight is the softmax of the row at it, over all experts
// or over the choices.  The T k choices are then ordered by (expert, token):
// the slot of a choice is the number of choices of earlier experts, plus that
// of earlier tokens' choices of the same expert.  A token chooses an expert at
// most once, so among 64 tokens the choices of an expert are a 64-bit mask,
// and a choice's place among them is the number of bits below its own: the
// order does not depend on when an atomic lands.
//
// Bound by the choices' chains of instructions, not by the bytes (2 MB for 8192 tokens of
// 64 experts in bf16, which take 6.0 us to choose 8 each from and 4.9 to place).
//
// Of few tokens one workgroup does it all (16 tokens, 4 of 128: 4.4 us).  Above, one kernel chooses, 32
// tokens a workgroup (a wave takes two), and counts the choices of every expert
// in them, and a second one adds up what stands before each 64 tokens and
// places them.  Where that sum is
// long (kMaxCounts) a kernel between the two turns the counts into sums.
#include "experts.h"
#include "wide_types.h"

#include <algorithm>
#include <cmath>

namespace cnn {
namespace {

constexpr int kTokens = 32;      // tokens a workgroup, where there are several
constexpr int kOne = 64;         // tokens that a workgroup places, and the most up to which one does it all
constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;

// Reductions over the wave by data-parallel moves: rows of 16 lanes first, then
// across rows, the result in lane 63 and from there everywhere.  Lanes that a
// move reads nothing for give 0, which changes neither a maximum of
// unsigned values nor a sum.  (Through lane exchanges, which go by LDS, a
// token's eight maxima took four times as long.)
template <int CTRL, int ROWS>
__device__ inline unsigned moved(unsigned v) {
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, true);
}
__device__ inline unsigned wave_umax(unsigned v) {
    v = max(v, moved<0x111, 0xf>(v));  // one lane up
    v = max(v, moved<0x112, 0xf>(v));
    v = max(v, moved<0x114, 0xf>(v));
    v = max(v, moved<0x118, 0xf>(v));
    v = max(v, moved<0x142, 0xa>(v));  // lane 15 of a row to the next row, 1 and 3
    v = max(v, moved<0x143, 0xc>(v));  // lane 31 to rows 2 and 3
    return (unsigned)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ inline float wave_sum(float f) {
    auto add = [](float a, unsigned b) { return a + __uint_as_float(b); };
    f = add(f, moved<0x111, 0xf>(__float_as_uint(f)));
    f = add(f, moved<0x112, 0xf>(__float_as_uint(f)));
    f = add(f, moved<0x114, 0xf>(__float_as_uint(f)));
    f = add(f, moved<0x118, 0xf>(__float_as_uint(f)));
    f = add(f, moved<0x142, 0xa>(__float_as_uint(f)));
    f = add(f, moved<0x143, 0xc>(__float_as_uint(f)));
    return __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(f), 63));
}

// A number that orders as the logit does, -0 as 0; 0 for what is never chosen (minus
// infinity and NaN) or not `there`.  Without branches: a token has up to 16 a lane.
__device__ inline unsigned order_key(float v, bool there) {
    const unsigned u = __float_as_uint(v + 0.0f);
    return (u ^ ((unsigned)((int)u >> 31) | 0x80000000u)) & -(unsigned)(there & (v > -INFINITY));
}
__device__ inline float key_logit(unsigned key) {
    return __uint_as_float((key >> 31) ? key & 0x7fffffffu : ~key);
}

// One wave, one token: lane l holds experts l, l + 64, ... (J of them, as
// order keys).  Lane c ends up with choice c.
template <int J>
__device__ inline void choose(unsigned (&key)[J], int k, bool renorm, int32_t* expert, float* weight,
                              unsigned long long* mask, int bit) {
    const int lane = threadIdx.x & 63;
    unsigned best[J], mine = 0;  // best: of key[0..j], kept up as keys go
    int my_expert = -1;
    float sum = 0.0f, top = 0.0f;
    for (int c = 0; c < k; ++c) {
        best[0] = key[0];
#pragma unroll
        for (int j = 1; j < J; ++j) best[j] = max(best[j - 1], key[j]);
        const unsigned most = wave_umax(best[J - 1]);
        if (most == 0) break;  // nothing left that may be chosen
        int e = 0;
#pragma unroll
        for (int j = J - 1; j >= 0; --j) {
            const unsigned long long at = __ballot(key[j] == most);
            if (at) e = 64 * j + __builtin_ctzll(at);
        }
        if (c == 0) {
            top = key_logit(most);
            if (!renorm) {
#pragma unroll
                for (int j = 0; j < J; ++j)
                    sum += expf(key[j] ? key_logit(key[j]) - top : -INFINITY);
            }
        }
        if (lane == c) {
            mine = most;
            my_expert = e;
        }
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (e == lane + 64 * j) key[j] = 0;
    }
    const float p = mine ? expf(key_logit(mine) - top) : 0.0f;
    sum = wave_sum(renorm ? p : sum);
    if (lane < k) {
        expert[lane] = my_expert;
        weight[lane] = mine ? p / sum : 0.0f;
        if (mine) atomicOr(&mask[my_expert], 1ull << bit);
    }
}

struct RouteParams {
    const void* logits;
    int T, E, k, renorm;
    int32_t* expert;
    float* weight;
    int32_t* rows;
    int32_t* offsets;
    int32_t* slot;
    int32_t* counts;  // [ceil(T / 32)][E], and the totals
};

// The experts of the choices of n <= kOne tokens from t0 on, of this work-item:
// choices threadIdx.x, + kThreads, ...
constexpr int kMostChoices = 64;
struct Choices {
    static constexpr int kEach = kOne * kMostChoices / kThreads;
    int expert[kEach];

    __device__ void load(const RouteParams& p, int t0, int n) {
#pragma unroll
        for (int c = 0; c < kEach; ++c) {
            const int i = threadIdx.x + c * kThreads;
            expert[c] = i < n * p.k ? p.expert[(size_t)t0 * p.k + i] : -1;
        }
    }
    // Marks the tokens in their experts' masks.
    __device__ void mark(const RouteParams& p, unsigned long long* mask) const {
#pragma unroll
        for (int c = 0; c < kEach; ++c)
            if (expert[c] >= 0) atomicOr(&mask[expert[c]], 1ull << ((threadIdx.x + c * kThreads) / (unsigned)p.k));
    }
    // first[e]: the slot of the first of these tokens' choices of expert e.
    __device__ void place(const RouteParams& p, int t0, int n, const int* first, const unsigned long long* mask) const {
#pragma unroll
        for (int c = 0; c < kEach; ++c) {
            const int i = threadIdx.x + c * kThreads;
            if (i >= n * p.k) break;
            const int t = (int)((unsigned)i / (unsigned)p.k), e = expert[c];
            int s = -1;
            if (e >= 0) {
                s = first[e] + __builtin_popcountll(mask[e] & ((1ull << t) - 1));
                p.rows[s] = t0 + t;
            }
            p.slot[(size_t)t0 * p.k + i] = s;
        }
    }
};

// before[e] = sum of total[e'] over e' < e, in LDS, and the sum of all in
// *sum; the first wave does it.
__device__ inline void scan_experts(const int* total, int* before, int E, int* sum) {
    if (threadIdx.x < 64) {
        int run = 0;
        for (int base = 0; base < E; base += 64) {
            const int e = base + (int)threadIdx.x;
            const int v = e < E ? total[e] : 0;
            int incl = v;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const int u = __shfl_up(incl, off);
                if ((int)threadIdx.x >= off) incl += u;
            }
            if (e < E) before[e] = run + incl - v;
            run += __shfl(incl, 63);
        }
        if (threadIdx.x == 0) *sum = run;
    }
}

// ONE: all tokens are this workgroup's, which places them too.
template <typename T, int J, bool ONE>
__global__ void __launch_bounds__(kThreads) route_choose(RouteParams p) {
    constexpr int MOST = ONE ? kOne : kTokens, EACH = MOST / kWaves;  // tokens a wave
    __shared__ unsigned long long mask[64 * J];
    __shared__ int total[64 * J], before[64 * J], sum;
    const int t0 = blockIdx.x * MOST, lane = threadIdx.x & 63;
    const int n = min(MOST, p.T - t0);
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    // all of the wave's logits are on their way before the first token's choices
    T logit[EACH][J];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const T* row = (const T*)p.logits + (size_t)(t0 + min(wave + i * kWaves, n - 1)) * p.E;
#pragma unroll
        for (int j = 0; j < J; ++j) logit[i][j] = row[min(lane + 64 * j, p.E - 1)];
    }
    unsigned key[EACH][J];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
#pragma unroll
        for (int j = 0; j < J; ++j) key[i][j] = order_key(to_f32(logit[i][j]), lane + 64 * j < p.E);
    }
    for (int e = threadIdx.x; e < p.E; e += kThreads) mask[e] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int t = wave + i * kWaves;
        const size_t row = (size_t)(t0 + t);
        if (t < n) choose<J>(key[i], p.k, p.renorm != 0, p.expert + row * p.k, p.weight + row * p.k, mask, t);
    }
    __syncthreads();
    if constexpr (ONE) {
        for (int e = threadIdx.x; e < p.E; e += kThreads) total[e] = __builtin_popcountll(mask[e]);
        __syncthreads();
        scan_experts(total, before, p.E, &sum);
        __syncthreads();
        for (int e = threadIdx.x; e < p.E; e += kThreads) p.offsets[e] = before[e];
        if (threadIdx.x == 0) p.offsets[p.E] = sum;
        Choices mine;
        mine.load(p, 0, n);
        mine.place(p, 0, n, before, mask);
        for (int i = sum + (int)threadIdx.x; i < n * p.k; i += kThreads) p.rows[i] = -1;
    } else {
        for (int e = threadIdx.x; e < p.E; e += kThreads)
            p.counts[(size_t)blockIdx.x * p.E + e] = __builtin_popcountll(mask[e]);
    }
}

// Counts to the sums of the workgroups before, in place; the row behind
// the last workgroup's gets the totals.  A workgroup takes 64 experts, its
// waves consecutive runs of the rows.
__global__ void __launch_bounds__(kThreads) route_scan(int32_t* counts, int groups, int E) {
    __shared__ int part[kWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int e = blockIdx.x * 64 + lane;
    const int64_t run = (groups + kWaves - 1) / kWaves;
    const int64_t lo = std::min<int64_t>(wave * run, groups), hi = std::min<int64_t>(lo + run, groups);
    int s = 0;
    if (e < E) {
#pragma unroll 8
        for (int64_t g = lo; g < hi; ++g) s += counts[g * E + e];
    }
    part[wave][lane] = s;
    __syncthreads();
    if (e >= E) return;
    int at = 0;
    for (int w = 0; w < wave; ++w) at += part[w][lane];
    constexpr int BATCH = 8;  // loads on their way before the first store
    for (int64_t g = lo; g < hi; g += BATCH) {
        int v[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) v[i] = g + i < hi ? counts[(g + i) * E + e] : 0;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            if (g + i < hi) counts[(g + i) * E + e] = at;
            at += v[i];
        }
    }
    if (wave == kWaves - 1) counts[(int64_t)groups * E + e] = at;
}

// SCANNED: counts hold the sums of route_scan.  A workgroup places the choices
// of kOne tokens, those of kOne / kTokens rows of counts.
template <bool SCANNED>
__global__ void __launch_bounds__(kThreads) route_place(RouteParams p, int groups) {
    __shared__ unsigned long long mask[1024];
    __shared__ int total[1024], mine[1024], before[1024], sum;
    const int t0 = blockIdx.x * kOne, g0 = blockIdx.x * (kOne / kTokens);
    const int n = min(kOne, p.T - t0);
    Choices choices;
    choices.load(p, t0, n);
    for (int e = threadIdx.x; e < p.E; e += kThreads) {
        mask[e] = 0;
        if constexpr (SCANNED) {
            mine[e] = p.counts[(size_t)g0 * p.E + e];
            total[e] = p.counts[(size_t)groups * p.E + e];
        } else {
            mine[e] = total[e] = 0;
        }
    }
    __syncthreads();
    if constexpr (!SCANNED) {
        // work-item i adds up every so-manieth row of counts of expert i % E
        const int lanes = kThreads / p.E;  // at least 1: E <= 1024
        const int e = (int)threadIdx.x % p.E, r = (int)threadIdx.x / p.E;
        if (r < lanes) {
            int all = 0, earlier = 0;
#pragma unroll 8
            for (int g = r; g < groups; g += lanes) {
                const int v = p.counts[(size_t)g * p.E + e];
                all += v;
                earlier += g < g0 ? v : 0;
            }
            atomicAdd(&total[e], all);
            atomicAdd(&mine[e], earlier);
        }
    }
    choices.mark(p, mask);
    __syncthreads();
    scan_experts(total, before, p.E, &sum);
    __syncthreads();
    if (blockIdx.x == 0) {
        for (int e = threadIdx.x; e < p.E; e += kThreads) p.offsets[e] = before[e];
        if (threadIdx.x == 0) p.offsets[p.E] = sum;
    }
    for (int e = threadIdx.x; e < p.E; e += kThreads) mine[e] += before[e];
    __syncthreads();
    choices.place(p, t0, n, mine, mask);
    // this workgroup's share of the slots that no choice has
    const int64_t lo = std::max<int64_t>((int64_t)t0 * p.k, sum), hi = (int64_t)(t0 + n) * p.k;
    for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) p.rows[i] = -1;
}

__global__ void __launch_bounds__(kThreads) route_empty(int32_t* offsets, int E) {
    for (int e = threadIdx.x; e <= E; e += kThreads) offsets[e] = 0;
}

// Above this many counts every workgroup of route_place would read more than
// 128 KiB of them.
constexpr int64_t kMaxCounts = 32768;

// One workgroup's waves choose for a token each at a time, in a time that grows with the
// experts: 64 tokens take 6.3 us of 8 experts (two kernels 6.8), 9.8 of 64 (8.7) and 16.4 of
// 256 (12.4); 16 tokens 4.0, 4.9 and 7.3.
bool one_workgroup(int T, int E) { return T <= (E <= 32 ? kOne : E <= 128 ? 48 : 32); }

template <typename T, int J>
void run_route(const RouteParams& p, hipStream_t st) {
    const int groups = ceil_div(p.T, kTokens);
    if (one_workgroup(p.T, p.E)) {
        enqueue(route_choose<T, J, true>, dim3(1), dim3(kThreads), 0, st, p);
        return;
    }
    enqueue(route_choose<T, J, false>, dim3(groups), dim3(kThreads), 0, st, p);
    if ((int64_t)groups * p.E <= kMaxCounts) {
        enqueue(route_place<false>, dim3(ceil_div(p.T, kOne)), dim3(kThreads), 0, st, p, groups);
    } else {
        enqueue(route_scan, dim3(ceil_div(p.E, 64)), dim3(kThreads), 0, st, p.counts, groups, p.E);
        enqueue(route_place<true>, dim3(ceil_div(p.T, kOne)), dim3(kThreads), 0, st, p, groups);
    }
}

template <typename T>
void run_route_type(const RouteParams& p, hipStream_t st) {
    if (p.E <= 64) run_route<T, 1>(p, st);
    else if (p.E <= 128) run_route<T, 2>(p, st);
    else if (p.E <= 256) run_route<T, 4>(p, st);
    else if (p.E <= 512) run_route<T, 8>(p, st);
    else run_route<T, 16>(p, st);
}

// Combine: y[t, d] = sum_j weight[t, j] x[slot[t, j], d], sums in fp32, j
// ascending.  Moves bytes and little else: a work-item takes 16 bytes of
// a row of y and so 16 bytes of each of its k rows of x (bf16, 4096 tokens of 8 rows of
// 2048: 30 to 32 us, 4.7 to 5.0 TB/s; odd widths, whose vectors begin at any
// element, take a sixth more).
template <typename T>
__global__ void __launch_bounds__(256)
combine_rows(const T* x, int M, int D, const int32_t* slot, const float* weight, unsigned items, int k, T* y,
             int chunks, FastDiv f_chunks) {
    constexpr int N = 16 / (int)sizeof(T);
    const unsigned step = gridDim.x * 256;  // items and a step below 2^31: no wrap
    for (unsigned i = blockIdx.x * 256 + threadIdx.x; i < items; i += step) {
        const int64_t t = fdiv(i, f_chunks);
        const int d = (int)(i - (unsigned)t * chunks) * N;
        const bool whole = d <= D - N;  // d + N can be 2^31
        float acc[N];
#pragma unroll
        for (int c = 0; c < N; ++c) acc[c] = 0.0f;
        for (int j = 0; j < k; ++j) {
            const int s = slot[t * k + j];
            if (s < 0 || s >= M) continue;
            const float wt = weight[t * k + j];
            const T* src = x + (size_t)s * D + d;
            T part[N];
            if (whole) {
                const u32x4 u = load16(src);
                __builtin_memcpy(part, &u, 16);
            } else {
#pragma unroll
                for (int c = 0; c < N; ++c) part[c] = d + c < D ? src[c] : (T)0.0f;
            }
#pragma unroll
            for (int c = 0; c < N; ++c) acc[c] = fmaf(wt, to_f32(part[c]), acc[c]);
        }
        T* dst = y + (size_t)t * D + d;
        if (whole) {
            T part[N];
#pragma unroll
            for (int c = 0; c < N; ++c) part[c] = from_f32<T>(acc[c]);
            u32x4 u;
            __builtin_memcpy(&u, part, 16);
            store16(dst, u);
        } else {
#pragma unroll
            for (int c = 0; c < N; ++c)
                if (d + c < D) dst[c] = from_f32<T>(acc[c]);
        }
    }
}

template <typename T>
void run_combine(const T* x, int M, int D, const int32_t* slot, const float* weight, int N, int k, T* y, hipStream_t st) {
    const int chunks = ceil_div(D, 16 / (int)sizeof(T));
    const unsigned items = (unsigned)N * chunks;  // no more than the elements of y
    enqueue(combine_rows<T>, dim3((unsigned)std::min<int64_t>(ceil_div64(items, 256), 1 << 20)), dim3(256), 0, st, x, M,
            D, slot, weight, items, k, y, chunks, make_fastdiv(chunks));
}

}  // namespace

size_t route_workspace(int T, int E) {
    const int64_t groups = ceil_div(T, kTokens);
    return one_workgroup(T, E) ? 0 : (size_t)(groups + 1) * E * sizeof(int32_t);
}

int launch_route(const void* logits, int type, int T, int E, int k, int renorm, int32_t* expert, float* weight,
                 int32_t* rows, int32_t* offsets, int32_t* slot, int32_t* counts, hipStream_t st) {
    if (T == 0) {
        enqueue(route_empty, dim3(1), dim3(kThreads), 0, st, offsets, E);
        return check_launch("route_empty");
    }
    const RouteParams p{logits, T, E, k, renorm, expert, weight, rows, offsets, slot, counts};
    if (type == CNN_F32) run_route_type<float>(p, st);
    else if (type == CNN_BF16) run_route_type<bf16_t>(p, st);
    else run_route_type<f16_t>(p, st);
    return check_launch("route");
}

int launch_combine(const void* x, int type, int M, int D, const int32_t* slot, const float* weight, int N, int k,
                   void* y, hipStream_t st) {
    if (N == 0) return CNN_OK;
    if (type == CNN_F32) run_combine((const float*)x, M, D, slot, weight, N, k, (float*)y, st);
    else if (type == CNN_BF16) run_combine((const bf16_t*)x, M, D, slot, weight, N, k, (bf16_t*)y, st);
    else run_combine((const f16_t*)x, M, D, slot, weight, N, k, (f16_t*)y, st);
    return check_launch("combine_rows");
}

}  // namespace cnn
