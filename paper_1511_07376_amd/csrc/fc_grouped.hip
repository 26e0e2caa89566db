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

// Up to 16 rows a group (on average: offsets are on the device) the weights
// are streamed.  A plain layer on 4-bit weights, whose rows are known, up to 32 (24 rows,
// 4096 x 4096, bf16: 9.6 us against 18.8 on tiles), but for inputs in fp32, whose parts
// are then cut once for every 16 outputs (32 rows, 9216 x 4096: 42 us against 31).
bool few_rows(const GroupedFc& p) {
    const bool wide_pass = !p.offsets && p.w_type == CNN_MX4 && p.x_type != CNN_F32;
    return ceil_div64(p.M, p.G) <= (wide_pass ? 32 : 16);
}

// Whole 16-byte vectors: rows of wide operands that begin and end at one.
bool whole_vectors(const GroupedFc& p) {
    auto whole = [&](const void* base, int type) {
        return type == CNN_MX4 || ((uintptr_t)base % 16 == 0 && (int64_t)p.I * type_bytes(type) % 16 == 0);
    };
    return whole(p.x, p.x_type) && whole(p.w, p.w_type);
}

// Inputs that are cut into parts beside 4-bit weights.
bool cut_inputs(const GroupedFc& p) { return p.w_type == CNN_MX4 && (p.x_type == CNN_F32 || p.x_type == CNN_F16); }

// Of the smallest tiles the fp32 ones are bound by the matrix cores at any number of
// rows: 32 rows up to 64 a group (128 tokens, 4 of 16 experts of 2048 x 2048: 85 us
// against 150 on 64 rows), 64 above (900 tokens, 2 of 4 of 1000 x 2000: 78 against 90).
//
// A slab's nanoseconds with two workgroups a compute unit were measured between
// reductions of 4096 and 9216 values, 64 rows: fp32 inputs that are cut 1150, fp16 ones
// 800, bf16 beside 4-bit weights 475, 4 bits both 660.  Larger tiles take about as much
// more as they have products a wave (256 x 256 in bf16: 1750).  One workgroup alone
// is no faster (share 0.5: it waits half the time), but in fp32, where two take 1.1
// (32 rows) to 1.7 times as long.  Writing and joining a part: 0.65 us a MB.
TileSize tile_size(const GroupedFc& p, int index) {
    const bool cut = cut_inputs(p), wide32 = p.w_type == CNN_F32, small32 = wide32 && ceil_div64(p.M, p.G) <= 64;
    const float ns = p.x_type == CNN_MX4 ? 660 : wide32 ? 1300 : !cut ? 475 : p.x_type == CNN_F32 ? 1150 : 800;
    const float share = wide32 ? 0.85f : 0.5f;
    TileSize t;
    if (index == 0) t = small32 ? TileSize{0, 32, 128, 512, 0, 1200, 0.55f, 0} : TileSize{0, 64, 128, 512, 0, ns, share, 0};
    else if (index == 1) t = {1, 128, 128, 512, 0, 2 * ns, share, 0};
    else t = {2, cut ? 128 : 256, 256, 256, 0, (cut ? 2 : 4) * ns, 1, 0};
    t.room = std::min(2 * t.slots, (64 << 20) / (t.rows * t.outs * (int)sizeof(float)));  // no workspace above 64 MB
    t.part_ns = (float)(t.rows * t.outs) * 4 * 0.00065f;
    return t;
}

// By sizes and types alone (the workspace is sized before the call's pointers
// are known).  The larger tile where there are enough of them for all compute
// units: 2048 x 4096 x 4096 in bf16 on 4-bit weights 94, 77 and 106 us by size
// (512 of 128 x 128), 4096 x 8192 x 8192 644, 555 and 482 (512 of 256 x 256), 512
// tokens, 2 of 8 experts of 2048 x 2048 34, 38 and 56.  Cut inputs: each value is
// cut once a workgroup, so the one with the most outputs (256 x 9216 x 4096 76, 86 and 72).
int choose_size(const GroupedFc& p) {
    const int64_t each = ceil_div64(p.M, p.G);
    auto tiles = [&](int size) {
        const TileSize t = tile_size(p, size);
        return ceil_div64(each, t.rows) * p.G * ceil_div(p.O, t.outs);
    };
    if (each <= 64) return 0;
    if (cut_inputs(p)) return 2;
    if (p.x_type != CNN_MX4 && (int64_t)p.I * type_bytes(p.x_type) % 16 == 0 && tiles(2) >= 256) return 2;
    return tiles(1) >= 384 ? 1 : 0;
}

// Whether the tail of this call's tiles is to be split: known without groups; with
// groups by their expected number, half a tile more than its rows for each.  Where
// it is not, the call is one kernel: 128 tokens, 4 of 16 experts of 2048 x 2048, bf16
// 41.9 us against 45.9 with a join that finds next to nothing to do.
bool may_split(const GroupedFc& p, const TileSize& size) {
    TileParams tp{};
    tp.cols = ceil_div(p.O, size.outs);
    tp.slabs = ceil_div(p.I, p.x_type == CNN_MX4 ? 256 : p.w_type == CNN_F32 ? 32 : 64);
    tp.unroll = 4;
    tp.slots = size.slots;
    tp.room = size.room;
    tp.slab_ns = size.slab_ns;
    tp.share = size.share;
    tp.part_ns = size.part_ns;
    const int64_t row_tiles = ceil_div64(p.M, size.rows) + (p.offsets ? std::min(p.G, p.M) / 2 : 0);
    return make_tail(tp, (int)std::min<int64_t>(row_tiles * tp.cols, INT32_MAX)).parts > 1;
}

// The parts that the workspace holds for a call's tiles: 0 if none is split.
int parts_held(const GroupedFc& p, const TileSize& size) {
    if (!may_split(p, size)) return 0;
    const int64_t tiles = (ceil_div64(p.M, size.rows) + (p.offsets ? p.G : 0)) * ceil_div(p.O, size.outs);
    return (int)std::min<int64_t>(size.room, tiles * kMaxParts);
}

}  // namespace

size_t fc_grouped_workspace(const GroupedFc& p) {
    if (p.M == 0 || few_rows(p)) return 0;
    const TileSize size = tile_size(p, choose_size(p));
    return (size_t)parts_held(p, size) * size.rows * size.outs * sizeof(float);
}

int launch_fc_grouped(const GroupedFc& p, float* ws, hipStream_t st) {
    if (p.M == 0) return CNN_OK;
    if (few_rows(p)) return run_fc_rows(p, st);
    const bool vec = whole_vectors(p);
    int index = choose_size(p);
    const size_t bytes = fc_grouped_workspace(p);
    // rows of whole vectors at an address that is none
    if (index == 2 && !vec && !cut_inputs(p)) index = 1;
    TileSize size = tile_size(p, index);
    size.room = std::min(parts_held(p, size), (int)(bytes / ((size_t)size.rows * size.outs * sizeof(float))));
    if (p.x_type == CNN_MX4) run_tiles_mx4(p, size, vec, ws, st);
    else if (p.w_type != CNN_MX4) p.x_type == CNN_F32 ? run_tiles_f32(p, size, vec, ws, st) : run_tiles_16(p, size, vec, ws, st);
    else if (p.x_type == CNN_BF16) run_tiles_wide_mx4(p, size, vec, ws, st);
    else run_tiles_cut(p, size, vec, ws, st);
    return check_launch("fc_tiles");
}

}  // namespace cnn
