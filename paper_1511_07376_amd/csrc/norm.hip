// Root-mean-square norm of rows, with the residual's addition before it and a
// result that may be 8-bit floats:
//
//     s = x + residual,  y[c] = s[c] / sqrt(mean(s^2) + eps) * weight[c]
//
// s is fp32 (it is rounded where it is stored, not where it is used), its squares
// are summed in 64 bits, which no value over- or underflows and which cost
// nothing beside the memory's time, y is rounded to fp32 after each product and then to its type.  8-bit
// results are made in 64 bits: a value near the middle between two 8-bit floats goes to the one
// that the definition gives, where fp32's roundings would now and then (a few of 10^7) take the other.
//
// Bound by HBM: every tensor is read or written once, a row held in registers
// between the sum and the result (up to 16384 values).  A work-item takes vectors of 8 values, so
// that 16 lanes hold a block of 128.  8192 x 4096 bf16 with residual and sum, to 8 bits: 59 to 63
// us, 3.9 TB/s, of which the 64 bits take 10 (made from fp32 values it was 50, 4.7 TB/s; a copy reaches
// 5.05); 77 x 1013 fp32 3 us, which is a kernel's least and a chain of load,
// sum and store.
#include "f8.h"

#include <algorithm>

namespace cnn {
namespace {

__device__ inline double wave_sum(double v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

// The sum over the workgroup, in every work-item.  `part`: 16 values of LDS that the call before
// the last one used.
__device__ inline double group_sum(double v, double* part) {
    v = wave_sum(v);
    const int waves = (int)(blockDim.x >> 6);
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
    for (int w = 1; w < waves; ++w) v += part[w];
    return v;
}

// The largest of 16 neighbouring lanes, in all of them: rotations within a row of 16.
template <int CTRL>
__device__ inline double rotated(double v) {
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    const unsigned lo = (unsigned)__builtin_amdgcn_mov_dpp((int)u, CTRL, 0xf, 0xf, true), hi = (unsigned)__builtin_amdgcn_mov_dpp((int)(u >> 32), CTRL, 0xf, 0xf, true);
    return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
__device__ inline double max_of_16_lanes(double v) {
    v = fmax(v, rotated<0x128>(v));
    v = fmax(v, rotated<0x124>(v));
    v = fmax(v, rotated<0x122>(v));
    return fmax(v, rotated<0x121>(v));
}

template <typename T, bool F8>
struct Output {
    T* y;
    uint8_t* q;
    float* scale;
    T* sum;
    // 8 results of a row from column c on (c: cols or more for lanes with none; all
    // 16 lanes of a block are here)
    __device__ void put(int row, int c, int cols, int blocks, const float* s, const float* w, double r) const {
        if (sum) store_values8(sum + (size_t)row * cols, c, cols, s);
        float v[8];
        if constexpr (F8) {
            // s w and its maximum are exact in 64 bits
            double p[8], top = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[i] = (double)s[i] * (double)w[i];  // 0 behind the row
                top = fmax(top, fabs(p[i]));
            }
            const double a = fmax(max_of_16_lanes(top) * r, (double)kF8LeastTop), factor = r * (double)(float)((double)kF8Most / a);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = c < cols - i ? (float)(p[i] * factor) : 0.0f;  // 0 over 0 too
            // (a value that is none makes its scaled one NaN: infinity is scaled by 0)
            const float of = (float)(a * (1 / (double)kF8Most));
            const bool bad = max_of_16_lanes(top_bits8(v)) >= 0x7f800000u || of == INFINITY;
            store_f8(q + (size_t)row * cols, c, cols, bad ? u32x2{0, 0} : to_f8(v));
            if ((threadIdx.x & 15) == 0 && c < cols) scale[(size_t)row * blocks + c / kF8Block] = bad ? __uint_as_float(0x7fc00000u) : of;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (float)((double)s[i] * r) * w[i];
            store_values8(y + (size_t)row * cols, c, cols, v);
        }
    }
};

template <typename T>
__device__ inline void load_sum8(const T* x, const T* res, size_t at, int c, int cols, float* s) {
    load_values8(x + at, c, cols, s);
    if (res) {
        float r[8];
        load_values8(res + at, c, cols, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] += r[i];
    }
}
__device__ inline void load_weight8(const float* w, int c, int cols, float* v) {
    if (w) {
        load_values8(w, c, cols, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 1.0f;
    }
}
__device__ inline double sum_of_squares(const float* s, double sum) {
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fma((double)s[i], (double)s[i], sum);
    return sum;
}

// Rows of at most NV vectors a work-item.  The weights stay in registers from row to row.
template <typename T, bool F8, int NV>
__global__ void __launch_bounds__(1024) rms_norm_rows(const T* x, const T* res, const float* w, Output<T, F8> out, int rows, int cols, float eps) {
    __shared__ double part[2][16];
    const int nt = blockDim.x, tid = threadIdx.x, blocks = (int)(((int64_t)cols + kF8Block - 1) / kF8Block);
    int at[NV];
    float wv[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        at[j] = min((tid + j * nt) * 8, cols);
        load_weight8(w, at[j], cols, wv[j]);
    }
    int turn = 0;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x, turn ^= 1) {
        float s[NV][8];
        double sq = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j) load_sum8(x, res, (size_t)row * cols, at[j], cols, s[j]);
#pragma unroll
        for (int j = 0; j < NV; ++j) sq = sum_of_squares(s[j], sq);
        const double r = 1.0 / sqrt(group_sum(sq, part[turn]) / cols + (double)eps);
#pragma unroll
        for (int j = 0; j < NV; ++j) out.put((int)row, at[j], cols, blocks, s[j], wv[j], r);
    }
}

// Longer rows: read twice, the second time mostly from the caches.  1024 x 32768 bf16 to 8 bits: 71 us, 3.3
// TB/s.  (Four vectors a work-item held in registers spill.)
// Each value is read before it is written, by the same work-item: y and sum may be x or residual.
template <typename T, bool F8>
__global__ void __launch_bounds__(1024) rms_norm_long(const T* x, const T* res, const float* w, Output<T, F8> out, int rows, int cols, float eps) {
    __shared__ double part[2][16];
    const int tid = threadIdx.x, blocks = (int)(((int64_t)cols + kF8Block - 1) / kF8Block);
    const int64_t end = ((int64_t)cols + 1023) / 1024 * 1024;  // whole blocks for the lanes
    int turn = 0;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x, turn ^= 1) {
        double sq = 0;
        for (int64_t c = (int64_t)tid * 8; c < cols; c += (int64_t)blockDim.x * 8) {
            float s[8];
            load_sum8(x, res, (size_t)row * cols, (int)c, cols, s);
            sq = sum_of_squares(s, sq);
        }
        const double r = 1.0 / sqrt(group_sum(sq, part[turn]) / cols + (double)eps);
        // from the end on, which the caches still hold
        for (int64_t c = (end - 1) / ((int64_t)blockDim.x * 8) * (blockDim.x * 8) + tid * 8; c >= 0; c -= (int64_t)blockDim.x * 8) {
            if (c >= end) continue;
            const int from = (int)min(c, (int64_t)cols);
            float s[8], wv[8];
            load_sum8(x, res, (size_t)row * cols, from, cols, s);
            load_weight8(w, from, cols, wv);
            out.put((int)row, from, cols, blocks, s, wv, r);
        }
    }
}

template <typename T, bool F8>
void run(const RmsNorm& p, hipStream_t st) {
    const Output<T, F8> out{(T*)p.y, (uint8_t*)p.y, p.y_scale, (T*)p.sum};
    const int64_t vectors = ceil_div64(p.cols, 8);
    const dim3 grid((unsigned)std::min(p.rows, 1 << 16));
    auto go = [&](auto kernel, int waves) {
        enqueue(kernel, grid, dim3(64 * waves), 0, st, (const T*)p.x, (const T*)p.residual, p.weight, out, p.rows, p.cols, p.eps);
    };
    const int64_t waves = ceil_div64(vectors, 64);
    // One vector a work-item up to 1024 work-items, of fp32 or to 8 bits up to 512: 4096 x 8192 took 77 us with one and 66 with
    // two in bf16 to 8 bits, 109 and 98 in fp32; 8192 x 4096 63 and 65, 97 and 101.  2048 x 16384 with two and read
    // twice: 72 and 74 in bf16 to 8 bits, 115 and 125 in fp32.
    if (waves <= (F8 || sizeof(T) == 4 ? 8 : 16)) go(rms_norm_rows<T, F8, 1>, (int)waves);
    else if (waves <= 32) go(rms_norm_rows<T, F8, 2>, (int)ceil_div64(waves, 2));
    else go(rms_norm_long<T, F8>, 16);
}

}  // namespace

int launch_rms_norm(const RmsNorm& p, hipStream_t st) {
    if (p.rows == 0) return CNN_OK;
    auto both = [&](auto one) {
        using T = decltype(one);
        if (p.y_type == CNN_F8) run<T, true>(p, st);
        else run<T, false>(p, st);
    };
    if (p.type == CNN_F32) both(float{});
    else if (p.type == CNN_BF16) both(bf16_t{});
    else both(f16_t{});
    return check_launch("rms_norm");
}

}  // namespace cnn
