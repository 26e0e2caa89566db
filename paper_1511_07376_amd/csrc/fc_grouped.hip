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

TileSize tile_size(const GroupedFc& p, int size) {
    const bool cut = cut_inputs(p);
    if (size == 0) return {64, 128, 512};
    if (size == 1) return {128, 128, cut && p.x_type == CNN_F32 ? 256 : 512};
    return {cut ? 128 : 256, 256, 256};
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

}  // namespace

size_t fc_grouped_workspace(const GroupedFc& p) {
    if (p.M == 0 || few_rows(p)) return 0;
    const TileSize t = tile_size(p, choose_size(p));
    const int64_t tiles = (ceil_div64(p.M, t.rows) + (p.offsets ? p.G : 0)) * ceil_div(p.O, t.outs);
    // without groups the tail is known: half the slots or more are not split
    if (!p.offsets && tiles % t.slots * 2 > t.slots) return 0;
    if (!p.offsets && tiles % t.slots == 0) return 0;
    return (size_t)std::min<int64_t>(t.slots, tiles * kMaxParts) * t.rows * t.outs * sizeof(float);
}

int launch_fc_grouped(const GroupedFc& p, float* ws, hipStream_t st) {
    if (p.M == 0) return CNN_OK;
    if (few_rows(p)) return run_fc_rows(p, st);
    const bool vec = whole_vectors(p);
    int size = choose_size(p);
    float* partial = fc_grouped_workspace(p) > 0 ? ws : nullptr;
    // rows of whole vectors at an address that is none: the 128 x 128 tiles need no more workspace
    if (size == 2 && !vec && !cut_inputs(p)) size = 1;
    const int slots = tile_size(p, size).slots;
    if (p.x_type == CNN_MX4) run_tiles_mx4(p, size, slots, vec, partial, st);
    else if (p.w_type != CNN_MX4) p.x_type == CNN_F32 ? run_tiles_f32(p, size, slots, vec, partial, st) : run_tiles_16(p, size, slots, vec, partial, st);
    else if (p.x_type == CNN_BF16) run_tiles_wide_mx4(p, size, slots, vec, partial, st);
    else run_tiles_cut(p, size, slots, vec, partial, st);
    return check_launch("fc_tiles");
}

}  // namespace cnn
