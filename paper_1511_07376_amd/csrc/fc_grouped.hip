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

// Inputs that are cut into parts beside 4-bit weights.
bool cut_inputs(const GroupedFc& p) { return p.w_type == CNN_MX4 && (p.x_type == CNN_F32 || p.x_type == CNN_F16); }

// Few rows a group (on average: offsets are on the device, and what uneven groups cost the
// kernel says): the weights are streamed,
// once for every 16 rows, by many small workgroups.  Tiles take some 10 us at least, but read
// the weights once and feed the matrix cores better, so with more rows the
// streamed weights have to be few: of a plain layer on 4-bit weights up to 32 rows
// (4096 x 4096, 28 rows, bf16: 10.9 us against 12.0 on tiles; 8192 x 8192: 35.7
// against 17.8; 1000 outputs of 9216 values, too few workgroups: 20.7 against 12.1), of fp32
// inputs, whose parts are cut again for every 16 outputs, up to 16 (4096 x 4096, 16 rows:
// 12.3 against 14.5, 8192 x 8192: 39.4 against 25.9).  With groups up to 16 rows, as many of
// which have more than the average (16 of 16 rows, 2048 x 2048, fp32 184 against 80, bf16 58
// against 40, on 4-bit weights 25 against 22, 4 bits both 18 against 12.5; 64 of 12 rows of
// 2048 x 1024 cut to parts 67 against 48; 7 of 11 rows of 1000 x 720, bf16: 7.6 against
// 15.7), or the tiles themselves have to be few for all compute units (91 of 15 rows, 198 x
// 500, bf16 25 against 13, on 4-bit weights fp32 27 against 12).  fp32 products that take most of the matrix cores: up to 4 (16 groups of 5 rows: 102
// against 69).
bool few_rows(const GroupedFc& p) {
    const int64_t each = ceil_div64(p.M, p.G), weights = (int64_t)p.I * p.O * p.G;
    const bool wide32 = p.w_type == CNN_F32;
    if (each <= (wide32 ? 4 : 8)) return true;
    if (!p.offsets) {
        const bool small = p.I <= 6144 && weights <= 24 << 20;
        if (p.x_type == CNN_F32) return each <= 16 && small;
        return each <= 16 || (each <= 32 && (p.x_type == CNN_MX4 ? p.O <= 6144 : small));
    }
    const int64_t most = wide32 ? 8 : p.w_type != CNN_MX4 ? 32 : cut_inputs(p) ? 128 : 64;
    return each <= 16 && weights < most << 20 && (int64_t)p.G * ceil_div(p.O, 128) <= 320;
}

// Whole 16-byte vectors: rows of wide operands that begin and end at one.
bool whole_vectors(const GroupedFc& p) {
    auto whole = [&](const void* base, int type) {
        return type == CNN_MX4 || ((uintptr_t)base % 16 == 0 && (int64_t)p.I * type_bytes(type) % 16 == 0);
    };
    return whole(p.x, p.x_type) && whole(p.w, p.w_type);
}

// A slab's nanoseconds with two workgroups a compute unit were measured between
// reductions of 4096 and 9216 values, 64 rows: fp32 inputs that are cut 1150, fp16 ones
// 800, bf16 beside 4-bit weights 475, 4 bits both 660.  Larger tiles take about as much
// more as they have products a wave (256 x 256 in bf16: 1750), those of 32 rows 0.8.
// One workgroup alone is no faster (share 0.4 or 0.5: it waits half the time), but in
// fp32, where two take 1.1 (32 rows) to 1.7 times as long.  Writing and joining a part:
// 0.65 us a MB.
TileSize tile_of(const GroupedFc& p, int rows, int outs) {
    const bool wide32 = p.w_type == CNN_F32;
    const float ns = p.x_type == CNN_MX4 ? 660 : wide32 ? 1300 : !cut_inputs(p) ? 475 : p.x_type == CNN_F32 ? 1150 : 800;
    TileSize t{rows, outs, outs == 256 ? 256 : 512, 0, ns * (float)(rows * outs) / (64 * 128), wide32 ? 0.85f : 0.5f, 0};
    if (rows == 32) t.slab_ns = wide32 ? 1200 : 0.8f * ns, t.share = wide32 ? 0.55f : 0.4f;
    if (outs == 256) t.share = 1;
    t.part_ns = (float)(rows * outs) * 4 * 0.00065f;
    t.room = std::min(2 * t.slots, (64 << 20) / (rows * outs * (int)sizeof(float)));  // no workspace above 64 MB
    return t;
}

// By sizes and types alone (the workspace is sized before the call's pointers
// are known).
//
// Tiles of 32 rows where groups have few more: the matrix cores, which the types that take
// most of them are bound by, then work on fewer rows that are none (128 tokens, 4 of 16 experts
// of 2048 x 2048: fp32 85 us against 150 on 64 rows, on 4-bit weights fp32 38 against 56,
// bf16 22 against 25, bf16 on both sides 41.5 against 41.7).  With more rows a group (500
// tokens, 6 of 64: 47) on 4-bit weights fp32 74 against 81, bf16 35 against 33.  A plain
// layer's rows are known: two such tiles of 40 rows take more than one of 64 (4096
// x 4096, bf16: 15.9 against 15.2).  They are also the more workgroups in calls of
// little work altogether (600 tokens, 4 experts of 1000 x 1000: on 4-bit weights bf16
// 12.3 against 14.1, 4 bits both 7.9 against 8.7), but for 16 bits on both sides,
// which read the weights more often (100 tokens, 2 experts of 2000 x 4000: 28 against 24),
// and where larger ones are enough (1978 x 203 x 2496: 14.1 against 11.6).
// Cut inputs: 128 tokens, 9216 x 4096: 36.8 against 37.4 on 128 x 256, 700 tokens, 8 experts
// of 4096 x 4096 fp16 89 against 113, 1400 tokens 136 against 118: there each
// value is cut once a workgroup, so the one with the most outputs.
//
// Else the larger tile where there are enough of them for all compute units: 2048 x 4096 x
// 4096 in bf16 on 4-bit weights 94, 77 and 106 us by size (512 of 128 x 128), 512 tokens, 2
// of 8 experts of 2048 x 2048 34, 38 and 56.  256 x 256 of wide types where they also
// fill the last round of compute units (4096 x 4096 x 4096 on 4-bit weights 129 against 147
// on 128 x 128, 384 of them, 4096 x 2048 x 6144, 135 against 116), and with groups, whose
// last tiles are half empty, in two rounds or more of 1024 rows each (4096 tokens, 2 of 8
// experts of 4096 x 4096, bf16: 346 against 382; of 2048 x 2048 120 against 107; 8 of 64 of
// 2048 x 1024 234 against 222).  In fp32 64 rows pad less of groups up to 512 (700 tokens,
// 2 of 8 of 4096 x 4096: 474 against 533).
TileSize choose_size(const GroupedFc& p) {
    const int64_t each = ceil_div64(p.M, p.G);
    const bool little = (float)p.M * p.I * p.O <= 3e9f;
    auto tiles = [&](int rows, int outs) { return ceil_div64(each, rows) * p.G * ceil_div(p.O, outs); };
    if (cut_inputs(p)) return each <= 128 || little ? tile_of(p, 32, 128) : tile_of(p, 128, 256);
    const bool wide16 = p.w_type == CNN_BF16 || p.w_type == CNN_F16;
    if (each <= 32 || (little && !wide16 && tiles(32, 128) <= 512)) return tile_of(p, 32, 128);
    if (p.offsets && !wide16 && each <= (p.w_type == CNN_F32 ? 64 : 40)) return tile_of(p, 32, 128);
    if (each <= (p.w_type == CNN_F32 ? 512 : 64)) return tile_of(p, 64, 128);
    const int64_t most = tiles(256, 256), last = most % 256;
    const bool large = p.offsets ? each >= 1024 && most >= 512 : most >= 1024 || (most >= 256 && (last == 0 || last >= 192));
    if (p.x_type != CNN_MX4 && (int64_t)p.I * type_bytes(p.x_type) % 16 == 0 && large) return tile_of(p, 256, 256);
    return tiles(128, 128) >= 384 ? tile_of(p, 128, 128) : tile_of(p, 64, 128);
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
    const TileSize size = choose_size(p);
    return (size_t)parts_held(p, size) * size.rows * size.outs * sizeof(float);
}

int launch_fc_grouped(const GroupedFc& p, float* ws, hipStream_t st) {
    if (p.M == 0) return CNN_OK;
    if (few_rows(p)) return run_fc_rows(p, st);
    const bool vec = whole_vectors(p);
    TileSize size = choose_size(p);
    const size_t bytes = fc_grouped_workspace(p);
    // rows of whole vectors at an address that is none
    if (size.rows == 256 && !vec) size = tile_of(p, 128, 128);
    size.room = std::min(parts_held(p, size), (int)(bytes / ((size_t)size.rows * size.outs * sizeof(float))));
    if (p.x_type == CNN_MX4) run_tiles_mx4(p, size, vec, ws, st);
    else if (p.w_type != CNN_MX4) p.x_type == CNN_F32 ? run_tiles_f32(p, size, vec, ws, st) : run_tiles_16(p, size, vec, ws, st);
    else if (p.x_type == CNN_BF16) run_tiles_wide_mx4(p, size, vec, ws, st);
    else run_tiles_cut(p, size, vec, ws, st);
    return check_launch("fc_tiles");
}

}  // namespace cnn
