// Fully connected layers whose rows belong to groups with weights of their own
// (one group: a plain layer), and whose operands may be narrower than fp32:
//
//     y[m][o] = b[g][o] + sum_i x[rows[m]][i] * w[g][o][i],  offsets[g] <= m < offsets[g + 1]
//
// Sums are held in fp32 and rounded once, to the type of y.  Here: which kernel a
// call takes (by its sizes and types alone: offsets are on the device), and the sum of
// split reductions.
#include "fc_tiles_kernel.h"

#include <algorithm>

namespace cnn {
namespace {

// Adds the splits' sums in their order, then bias and ReLU, for the rows that
// are in a group.
template <int YT>
__global__ void __launch_bounds__(256) fc_join(GroupedFc p, const float* partial, int splits, int64_t units, int chunks) {
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int m = (int)(u / chunks);
        int g = -1;
        if (!p.offsets) {
            g = 0;
        } else {
            for (int base = 0; base < p.G && g < 0; base += 64) {
                const int e = base + (int)(threadIdx.x & 63);
                int lo = 0, hi = 0;
                if (e < p.G) group_rows(p.offsets, e, p.M, lo, hi);
                const unsigned long long in = __ballot(lo <= m && m < hi);
                if (in) g = base + __builtin_ctzll(in);
            }
            if (g < 0) continue;
        }
        const int64_t o = u % chunks * 256 + threadIdx.x;
        if (o >= p.O) continue;
        const size_t at = (size_t)m * p.O + o;
        float v = 0.0f;
        for (int s = 0; s < splits; ++s) v += partial[(size_t)s * p.M * p.O + at];
        if (p.bias) v += p.bias[(size_t)g * p.O + o];
        if (p.relu) v = v > 0.0f ? v : 0.0f;
        store_result<YT>(p.y, at, v);
    }
}

constexpr int kRowsMost = 16;  // average rows a group up to which the weights are streamed

bool few_rows(const GroupedFc& p) { return ceil_div64(p.M, p.G) <= kRowsMost; }

TilePlan plan_tiles(const GroupedFc& p) {
    const bool cut = p.w_type == CNN_MX4 && (p.x_type == CNN_F32 || p.x_type == CNN_F16);
    const int bk = p.x_type == CNN_MX4 ? 256 : p.x_type == CNN_F32 && p.w_type == CNN_F32 ? 32 : 64;
    const TileSize sizes[3] = {{64, 128}, {128, 128}, {cut ? 128 : 256, 256}};
    const int64_t each = ceil_div64(p.M, p.G);
    auto tiles = [&](int i) { return ceil_div64(each, sizes[i].rows) * p.G * ceil_div(p.O, sizes[i].outs); };
    const int size = each <= 64 ? 0 : tiles(2) >= 192 ? 2 : 1;
    const int64_t pairs = ceil_div64(ceil_div64(p.I, bk), 2);
    const int64_t want = std::max<int64_t>(1, 384 / tiles(size));
    const int64_t splits = std::min<int64_t>({want, std::max<int64_t>(1, pairs / 4), 16});
    const int64_t run = ceil_div64(pairs, splits);
    return TilePlan{size, (int)ceil_div64(pairs, run), (int)run};
}

}  // namespace

size_t fc_grouped_workspace(const GroupedFc& p) {
    if (p.M == 0 || few_rows(p)) return 0;
    const TilePlan plan = plan_tiles(p);
    return plan.splits > 1 ? (size_t)plan.splits * p.M * p.O * sizeof(float) : 0;
}

int launch_fc_grouped(const GroupedFc& p, float* ws, hipStream_t st) {
    if (p.M == 0) return CNN_OK;
    if (few_rows(p)) return run_fc_rows(p, st);
    const TilePlan plan = plan_tiles(p);
    // whole 16-byte vectors: rows of wide operands that begin and end at one
    auto whole = [&](const void* base, int type) {
        return type == CNN_MX4 || ((uintptr_t)base % 16 == 0 && (int64_t)p.I * type_bytes(type) % 16 == 0);
    };
    const bool vec = whole(p.x, p.x_type) && whole(p.w, p.w_type);
    if (p.x_type == CNN_MX4) run_tiles_mx4(p, plan, vec, ws, st);
    else if (p.w_type != CNN_MX4) p.x_type == CNN_F32 ? run_tiles_f32(p, plan, vec, ws, st) : run_tiles_16(p, plan, vec, ws, st);
    else if (p.x_type == CNN_BF16) run_tiles_wide_mx4(p, plan, vec, ws, st);
    else run_tiles_cut(p, plan, vec, ws, st);
    int rc = check_launch("fc_tiles");
    if (rc || plan.splits == 1) return rc;
    const int chunks = ceil_div(p.O, 256);
    const int64_t units = (int64_t)p.M * chunks;
    const dim3 grid((unsigned)std::min<int64_t>(units, 1 << 22));
    if (p.y_type == CNN_F32) enqueue(fc_join<CNN_F32>, grid, dim3(256), 0, st, p, (const float*)ws, plan.splits, units, chunks);
    else if (p.y_type == CNN_BF16) enqueue(fc_join<CNN_BF16>, grid, dim3(256), 0, st, p, (const float*)ws, plan.splits, units, chunks);
    else enqueue(fc_join<CNN_F16>, grid, dim3(256), 0, st, p, (const float*)ws, plan.splits, units, chunks);
    return check_launch("fc_join");
}

}  // namespace cnn
