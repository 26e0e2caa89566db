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
// Tokens are taken 64 to a workgroup (a wave takes four).  Up to 64 tokens,
// one workgroup does it all.  Above, one kernel chooses and counts the
// choices of every expert per 64 tokens, and a second one adds up what stands
// before each of its own 64 tokens and places them.  Where that sum is
// long (kMaxCounts) a kernel between the two turns the counts into sums.
#include "common.h"
#include "wide_types.h"

#include <algorithm>
#include <cmath>

namespace cnn {
namespace {

constexpr int kTokens = 64;      // tokens a workgroup
constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;

// Largest of the wave's values, in every lane.
__device__ inline unsigned wave_umax(unsigned v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = max(v, (unsigned)__shfl_xor((int)v, off));
    return v;
}
__device__ inline float wave_sum(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

// A number that orders as the logit does, -0 as 0; 0 for what is never chosen (minus
// infinity and NaN).
__device__ inline unsigned order_key(float v) {
    if (!(v > -INFINITY)) return 0;
    const unsigned u = __float_as_uint(v + 0.0f);
    return (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ inline float key_logit(unsigned key) {
    return __uint_as_float((key >> 31) ? key & 0x7fffffffu : ~key);
}

// One wave, one token: lane l holds experts l, l + 64, ... (J of them).
template <typename T, int J>
__device__ inline void choose(const T* row, int E, int k, bool renorm, int32_t* expert, float* weight,
                              unsigned long long* mask, int bit) {
    const int lane = threadIdx.x & 63;
    unsigned key[J];
#pragma unroll
    for (int j = 0; j < J; ++j) key[j] = lane + 64 * j < E ? order_key(to_f32(row[lane + 64 * j])) : 0;
    float top = 0.0f, all = 0.0f, chosen = 0.0f, mine = 0.0f;
    int my_expert = -1;
    for (int c = 0; c < k; ++c) {
        unsigned best = 0;
#pragma unroll
        for (int j = 0; j < J; ++j) best = max(best, key[j]);
        best = wave_umax(best);
        if (best == 0) break;  // nothing left that may be chosen
        int e = -1;
#pragma unroll
        for (int j = J - 1; j >= 0; --j) {
            const unsigned long long at = __ballot(key[j] == best);
            if (at) e = 64 * j + __builtin_ctzll(at);
        }
        const float logit = key_logit(best);
        if (c == 0) {
            top = logit;
            if (!renorm) {
                float s = 0.0f;
#pragma unroll
                for (int j = 0; j < J; ++j)
                    if (key[j]) s += expf(key_logit(key[j]) - top);
                all = wave_sum(s);
            }
        }
        const float p = expf(logit - top);
        chosen += p;
        if (lane == c) {
            mine = p;
            my_expert = e;
        }
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (e == lane + 64 * j) key[j] = 0;
    }
    if (lane < k) {
        expert[lane] = my_expert;
        weight[lane] = my_expert < 0 ? 0.0f : mine / (renorm ? chosen : all);
        if (my_expert >= 0) atomicOr(&mask[my_expert], 1ull << bit);
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
    int32_t* counts;  // [ceil(T / 64)][E]
};

// Places the choices of tokens [t0, t0 + n): first[e] is the slot of the first
// of these tokens' choices of expert e.
__device__ inline void place(const RouteParams& p, int t0, int n, const int* first, const unsigned long long* mask) {
    for (int i = threadIdx.x; i < n * p.k; i += kThreads) {
        const int t = i / p.k;
        const size_t at = (size_t)t0 * p.k + i;
        const int e = p.expert[at];
        int s = -1;
        if (e >= 0) {
            s = first[e] + __builtin_popcountll(mask[e] & ((1ull << t) - 1));
            p.rows[s] = t0 + t;
        }
        p.slot[at] = s;
    }
}

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
    __shared__ unsigned long long mask[64 * J];
    __shared__ int total[64 * J], before[64 * J], sum;
    const int t0 = blockIdx.x * kTokens;
    const int n = min(kTokens, p.T - t0);
    for (int e = threadIdx.x; e < p.E; e += kThreads) mask[e] = 0;
    __syncthreads();
    for (int t = (int)(threadIdx.x >> 6); t < n; t += kWaves) {
        const size_t row = (size_t)(t0 + t);
        choose<T, J>((const T*)p.logits + row * p.E, p.E, p.k, p.renorm != 0, p.expert + row * p.k,
                     p.weight + row * p.k, mask, t);
    }
    __syncthreads();
    if constexpr (ONE) {
        for (int e = threadIdx.x; e < p.E; e += kThreads) total[e] = __builtin_popcountll(mask[e]);
        __syncthreads();
        scan_experts(total, before, p.E, &sum);
        __syncthreads();
        for (int e = threadIdx.x; e < p.E; e += kThreads) p.offsets[e] = before[e];
        if (threadIdx.x == 0) p.offsets[p.E] = sum;
        place(p, 0, n, before, mask);
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
    if (e < E)
        for (int64_t g = lo; g < hi; ++g) s += counts[g * E + e];
    part[wave][lane] = s;
    __syncthreads();
    if (e >= E) return;
    int at = 0;
    for (int w = 0; w < wave; ++w) at += part[w][lane];
    for (int64_t g = lo; g < hi; ++g) {
        const int v = counts[g * E + e];
        counts[g * E + e] = at;
        at += v;
    }
    if (wave == kWaves - 1) counts[(int64_t)groups * E + e] = at;
}

// SCANNED: counts hold the sums of route_scan.
template <bool SCANNED>
__global__ void __launch_bounds__(kThreads) route_place(RouteParams p, int groups) {
    __shared__ unsigned long long mask[1024];
    __shared__ int total[1024], mine[1024], before[1024], sum;
    const int t0 = blockIdx.x * kTokens;
    const int n = min(kTokens, p.T - t0);
    for (int e = threadIdx.x; e < p.E; e += kThreads) {
        mask[e] = 0;
        if constexpr (SCANNED) {
            mine[e] = p.counts[(size_t)blockIdx.x * p.E + e];
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
            for (int g = r; g < groups; g += lanes) {
                const int v = p.counts[(size_t)g * p.E + e];
                all += v;
                earlier += g < (int)blockIdx.x ? v : 0;
            }
            atomicAdd(&total[e], all);
            atomicAdd(&mine[e], earlier);
        }
    }
    for (int i = threadIdx.x; i < n * p.k; i += kThreads) {
        const int e = p.expert[(size_t)t0 * p.k + i];
        if (e >= 0) atomicOr(&mask[e], 1ull << (i / p.k));
    }
    __syncthreads();
    scan_experts(total, before, p.E, &sum);
    __syncthreads();
    if (blockIdx.x == 0) {
        for (int e = threadIdx.x; e < p.E; e += kThreads) p.offsets[e] = before[e];
        if (threadIdx.x == 0) p.offsets[p.E] = sum;
    }
    for (int e = threadIdx.x; e < p.E; e += kThreads) mine[e] += before[e];
    __syncthreads();
    place(p, t0, n, mine, mask);
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

template <typename T, int J>
void run_route(const RouteParams& p, hipStream_t st) {
    const int groups = ceil_div(p.T, kTokens);
    if (groups == 1) {
        enqueue(route_choose<T, J, true>, dim3(1), dim3(kThreads), 0, st, p);
        return;
    }
    enqueue(route_choose<T, J, false>, dim3(groups), dim3(kThreads), 0, st, p);
    if ((int64_t)groups * p.E <= kMaxCounts) {
        enqueue(route_place<false>, dim3(groups), dim3(kThreads), 0, st, p, groups);
    } else {
        enqueue(route_scan, dim3(ceil_div(p.E, 64)), dim3(kThreads), 0, st, p.counts, groups, p.E);
        enqueue(route_place<true>, dim3(groups), dim3(kThreads), 0, st, p, groups);
    }
}

template <typename T>
void run_route_type(const RouteParams& p, hipStream_t st) {
    if (p.E <= 64) run_route<T, 1>(p, st);
    else if (p.E <= 128) run_route<T, 2>(p, st);
    else if (p.E <= 256) run_route<T, 4>(p, st);
    else run_route<T, 16>(p, st);
}

// Combine: y[t, d] = sum_j weight[t, j] x[slot[t, j], d], sums in fp32, j
// ascending.  Moves bytes and little else: a work-item takes 16 bytes of
// a row of y and so 16 bytes of each of its k rows of x.
template <typename T>
__global__ void __launch_bounds__(256)
combine_rows(const T* x, int M, int D, const int32_t* slot, const float* weight, int64_t items, int k, T* y,
             int chunks) {
    constexpr int N = 16 / (int)sizeof(T);
    const int64_t step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += step) {
        const int64_t t = i / chunks;
        const int d = (int)(i - t * chunks) * N;
        const bool whole = d + N <= D;
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
    const int64_t items = (int64_t)N * chunks;
    enqueue(combine_rows<T>, dim3((unsigned)std::min<int64_t>(ceil_div64(items, 256), 1 << 20)), dim3(256), 0, st, x, M,
            D, slot, weight, items, k, y, chunks);
}

}  // namespace

size_t route_workspace(int T, int E) {
    const int64_t groups = ceil_div(T, kTokens);
    return groups <= 1 ? 0 : (size_t)(groups + 1) * E * sizeof(int32_t);
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
