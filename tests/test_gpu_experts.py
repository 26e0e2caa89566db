"""Products grouped by expert, routing and combining (GPU), against references
in 64 bits (``experts_ref``), each by itself and run together as a block."""
import math

import pytest
import torch

import experts_ref as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
IDS = ["f32", "bf16", "f16"]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(shape, g, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def make_weights(kind, groups, o, i, g, dtype):
    """(w, w_scale, values in float64) of one kind of weights."""
    if kind == "mx4":
        w, ws = ref.random_mx4((groups, o), i, g)
        return w, ws, ref.values(w, ws, i)
    w = (randn((groups, o, i), g) / math.sqrt(i)).to(dtype)
    return w, None, w.double()


def check_grouped(y, x, wv, offsets, rows, bias, relu, what, untouched=None):
    """y against the reference, group by group; rows behind the last group hold `untouched`."""
    bounds = offsets.tolist()
    for g in range(len(bounds) - 1):
        lo, hi = bounds[g], bounds[g + 1]
        if lo == hi:
            continue
        src = torch.arange(lo, hi, device="cuda") if rows is None else rows[lo:hi].long()
        there = (src >= 0) & (src < x.shape[0])
        xg = torch.where(there.unsqueeze(1), x[src.clamp(0, x.shape[0] - 1)].double(), 0.0)
        want, s = ref.product(xg, wv[g], None if bias is None else bias[g], relu)
        ref.assert_product(y[lo:hi], want, s, x.shape[1], f"{what} group {g}")
    if untouched is not None:
        assert bool((y[bounds[-1]:] == untouched).all()), f"{what}: rows of no group were written"


SIZES = {
    "few_each": [1, 0, 2, 1, 3, 0],
    "ragged": [0, 5, 17, 0, 1, 64, 33],
    "one_has_all": [0, 0, 200, 0],
    "large": [130, 1, 256, 300, 0, 77],
    "single_group": [45],
    "none": [0, 0, 0],
}


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("kind", ["wide", "mx4"])
@pytest.mark.parametrize("i,o", [(64, 96), (610, 188), (33, 7), (256, 300)])
@pytest.mark.parametrize("sizes", list(SIZES.values()), ids=list(SIZES))
def test_fc_grouped(gpu, dtype, kind, i, o, sizes):
    g = gen(i + o + len(sizes))
    w, ws, wv = make_weights(kind, len(sizes), o, i, g, dtype)
    b = 0.1 * randn((len(sizes), o), g)
    m = sum(sizes)
    offsets = ints([0] + list(torch.tensor(sizes).cumsum(0)))
    # gathered from fewer rows than there are, with repetitions; 3 rows of y are in no group
    n = max(1, m // 2)
    x = randn((n, i), g, dtype)
    rows = torch.randint(0, n, (m + 3,), generator=g, device="cuda", dtype=torch.int32)
    y = torch.full((m + 3, o), -5.0, device="cuda", dtype=dtype)
    assert gpu.cnn_fc_grouped_fwd(x, w, offsets, b, True, rows=rows, w_scale=ws, y=y) is y
    check_grouped(y, x, wv, offsets, rows, b, True, f"{dtype} {kind} gathered", untouched=-5.0)
    # in place of the gather, row m of x; no bias
    x = randn((m, i), g, dtype)
    y = gpu.cnn_fc_grouped_fwd(x, w, offsets, w_scale=ws)
    assert y.shape == (m, o) and y.dtype == dtype
    check_grouped(y, x, wv, offsets, None, None, False, f"{dtype} {kind}")


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("kind", ["wide", "mx4"])
@pytest.mark.parametrize("sizes,i,o", [([3000, 0, 1300], 272, 6200), ([2300, 1], 1032, 2300), ([700, 400, 0, 900], 101, 3000)])
def test_fc_grouped_large(gpu, dtype, kind, sizes, i, o):
    """Rows and outputs for the larger tiles, the last of them split along the reduction; weights at an address that
    is aligned to their elements only."""
    g = gen(i + o)
    w, ws, wv = make_weights(kind, len(sizes), o, i, g, dtype)
    b = 0.1 * randn((len(sizes), o), g)
    m = sum(sizes)
    offsets = ints([0] + list(torch.tensor(sizes).cumsum(0)))
    x = randn((m // 3, i), g, dtype)
    rows = torch.randint(-1, m // 3, (m + 5,), generator=g, device="cuda", dtype=torch.int32)
    y = torch.full((m + 5, o), 2.0, device="cuda", dtype=dtype)
    gpu.cnn_fc_grouped_fwd(x, w, offsets, b, True, rows=rows, w_scale=ws, y=y)
    check_grouped(y, x, wv, offsets, rows, b, True, f"{dtype} {kind}", untouched=2.0)
    if kind == "wide":
        flat = torch.empty(w.numel() + 1, dtype=dtype, device="cuda")
        flat[1:] = w.reshape(-1)
        again = gpu.cnn_fc_grouped_fwd(x, flat[1:].view(w.shape), offsets, b, True, rows=rows)
        check_grouped(again, x, wv, offsets, rows, b, True, f"{dtype} unaligned")


@pytest.mark.parametrize("kind", ["wide", "mx4"])
@pytest.mark.parametrize("each,i", [(2, 200), (12, 1000), (30, 4096), (100, 2048), (200, 4096)])
def test_fc_grouped_rows_before_the_first_group(gpu, kind, each, i):
    """Groups that begin behind the first row and end before the last: the rows outside keep what they hold."""
    g = gen(each)
    o = 200
    w, ws, wv = make_weights(kind, 3, o, i, g, torch.float32)
    m, first = 3 * each + 12, 5
    offsets = ints([first, first + each, first + each, first + 3 * each])
    x = randn((m, i), g)
    y = torch.full((m, o), 7.0, device="cuda")
    gpu.cnn_fc_grouped_fwd(x, w, offsets, w_scale=ws, y=y)
    check_grouped(y, x, wv, offsets, None, None, False, f"{kind} {each}", untouched=7.0)
    assert bool((y[:first] == 7.0).all())


def one_behind(t):
    """The same values, contiguous, one element behind an aligned address."""
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    flat[1:] = t.reshape(-1)
    return flat[1:].view(t.shape)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("kind", ["wide", "mx4"])
@pytest.mark.parametrize("i", [1, 131, 517, 518, 1031, 4099])
@pytest.mark.parametrize("sizes", [[2, 1, 0, 4], [9, 0, 7, 12], [6] * 9], ids=["thin", "few", "even"])
def test_fc_grouped_few_rows_at_odd_addresses(gpu, dtype, kind, i, sizes):
    """Rows that begin at any element, in streams of weights: the values beside them are NaN and infinite."""
    g = gen(i + len(sizes))
    o = 77
    w, ws, wv = make_weights(kind, len(sizes), o, i, g, dtype)
    m = sum(sizes)
    offsets = ints([0] + list(torch.tensor(sizes).cumsum(0)))
    x = randn((m, i), g, dtype)
    want = gpu.cnn_fc_grouped_fwd(x, w, offsets, w_scale=ws)
    check_grouped(want, x, wv, offsets, None, None, False, f"{dtype} {kind}")
    for beside in (math.nan, math.inf):
        def between(t):
            flat = torch.full((t.numel() + 2,), beside, dtype=t.dtype, device="cuda")
            flat[1:-1] = t.reshape(-1)
            return flat[1:-1].view(t.shape)
        xo, wo = between(x), between(w) if kind == "wide" else w
        for a, b in ((xo, w), (x, wo), (xo, wo)):
            y = gpu.cnn_fc_grouped_fwd(a, b, offsets, w_scale=ws)
            check_grouped(y, x, wv, offsets, None, None, False, f"{dtype} {kind} beside {beside}")


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("kind", ["wide", "mx4", "mx4 both"])
@pytest.mark.parametrize("sizes", [[1, 0, 3] * 60, [7, 0, 9, 20] * 30, [2, 5], [0, 11]], ids=["thin", "few", "thin2", "few2"])
@pytest.mark.parametrize("i,o", [(32, 270), (128, 270), (129, 270), (256, 100), (500, 270), (513, 270), (1024, 100), (1025, 270)])
def test_fc_grouped_short_reductions(gpu, dtype, kind, sizes, i, o):
    """Reductions that a wave or two take, in many workgroups and in few."""
    g = gen(i + len(sizes))
    w, ws, wv = make_weights("wide" if kind == "wide" else "mx4", len(sizes), o, i, g, dtype)
    b = 0.1 * randn((len(sizes), o), g)
    m = sum(sizes)
    offsets = ints([0] + list(torch.tensor(sizes).cumsum(0)))
    if kind == "mx4 both":
        xq, xs = ref.random_mx4((m,), i, g)
        y = gpu.cnn_fc_grouped_fwd(xq, w, offsets, b, w_scale=ws, x_scale=xs, y_dtype=dtype)
        x = ref.values(xq, xs, i)
    else:
        x = randn((m, i), g, dtype)
        y = gpu.cnn_fc_grouped_fwd(x, w, offsets, b, w_scale=ws)
    check_grouped(y, x, wv, offsets, None, b, False, f"{dtype} {kind}")


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("kind", ["wide", "mx4", "mx4 both"])
@pytest.mark.parametrize("sizes,i,o", [([17, 40, 0, 64, 31, 1, 33, 90], 610, 1013), ([33] * 3, 4136, 500), ([20, 25] * 40, 198, 600),
                                       ([150, 0, 90], 521, 300), ([16, 9, 40, 0, 15] * 20, 40, 500)])
def test_fc_grouped_some_rows_each(gpu, dtype, kind, sizes, i, o):
    """Groups of some tens of rows: tiles of 32, with and without a split reduction."""
    g = gen(i + o)
    both = kind == "mx4 both"
    w, ws, wv = make_weights("mx4" if both else kind, len(sizes), o, i, g, dtype)
    b = 0.1 * randn((len(sizes), o), g)
    m = sum(sizes)
    offsets = ints([0] + list(torch.tensor(sizes).cumsum(0)))
    rows = torch.randint(-1, m // 2, (m + 3,), generator=g, device="cuda", dtype=torch.int32)
    y = torch.full((m + 3, o), 4.0, device="cuda", dtype=dtype)
    if both:
        xq, xs = ref.random_mx4((m // 2,), i, g)
        gpu.cnn_fc_grouped_fwd(xq, w, offsets, b, True, rows=rows, w_scale=ws, x_scale=xs, y_dtype=dtype, y=y)
        x = ref.values(xq, xs, i)
    else:
        x = randn((m // 2, i), g, dtype)
        gpu.cnn_fc_grouped_fwd(x, w, offsets, b, True, rows=rows, w_scale=ws, y=y)
        again = gpu.cnn_fc_grouped_fwd(one_behind(x), one_behind(w) if kind == "wide" else w, offsets, b, True, rows=rows, w_scale=ws)
        check_grouped(again, x, wv, offsets, rows, b, True, f"{dtype} {kind} unaligned")
    check_grouped(y, x, wv, offsets, rows, b, True, f"{dtype} {kind}", untouched=4.0)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("kind", ["wide", "mx4"])
@pytest.mark.parametrize("each,i,o", [(125, 1024, 2100), (300, 2088, 2100), (575, 1536, 2100)])
def test_fc_grouped_tails_in_rounds(gpu, dtype, kind, each, i, o):
    """Tails of more tiles than half of what runs at once, split along the reduction; the number of tiles is not
    the expected one where groups are uneven."""
    for sizes in ([each] * 8, [each * 3, 0, 1, each * 4 - 1, 0, 0, each, 0]):
        g = gen(each)
        w, ws, wv = make_weights(kind, 8, o, i, g, dtype)
        b = 0.1 * randn((8, o), g)
        offsets = ints([0] + list(torch.tensor(sizes).cumsum(0)))
        m = sum(sizes)
        x = randn((m, i), g, dtype)
        y = gpu.cnn_fc_grouped_fwd(x, w, offsets, b, True, w_scale=ws)
        check_grouped(y, x, wv, offsets, None, b, True, f"{dtype} {kind} {sizes}")
        assert torch.equal(gpu.cnn_fc_grouped_fwd(x, w, offsets, b, True, w_scale=ws), y)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("kind", ["wide", "mx4"])
@pytest.mark.parametrize("sizes,i,o", [([2500, 0, 800], 136, 8800), ([1100, 1201, 999], 1096, 8800), ([1500, 1210, 1100], 2056, 8800), ([3810, 0, 0], 2056, 8800)])
def test_fc_grouped_largest(gpu, dtype, kind, sizes, i, o):
    """The largest tiles, in more than two rounds; operands at an address that is aligned to their elements only."""
    g = gen(i + o)
    w, ws, wv = make_weights(kind, 3, o, i, g, dtype)
    b = 0.1 * randn((3, o), g)
    m = sum(sizes)
    offsets = ints([0] + list(torch.tensor(sizes).cumsum(0)))
    x = randn((m // 2, i), g, dtype)
    rows = torch.randint(-1, m // 2, (m + 2,), generator=g, device="cuda", dtype=torch.int32)
    y = torch.full((m + 2, o), 2.0, device="cuda", dtype=dtype)
    gpu.cnn_fc_grouped_fwd(x, w, offsets, b, True, rows=rows, w_scale=ws, y=y)
    check_grouped(y, x, wv, offsets, rows, b, True, f"{dtype} {kind}", untouched=2.0)
    del y
    again = gpu.cnn_fc_grouped_fwd(one_behind(x), w, offsets, b, True, rows=rows, w_scale=ws)
    check_grouped(again, x, wv, offsets, rows, b, True, f"{dtype} {kind} unaligned")


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("sizes", list(SIZES.values()), ids=list(SIZES))
@pytest.mark.parametrize("i,o", [(96, 64), (333, 190)])
def test_fc_grouped_of_mx4_inputs(gpu, dtype, sizes, i, o):
    g = gen(i + o)
    m = sum(sizes)
    n = max(1, m // 2)
    w, ws, wv = make_weights("mx4", len(sizes), o, i, g, dtype)
    xq, xs = ref.random_mx4((n,), i, g)
    b = 0.1 * randn((len(sizes), o), g)
    offsets = ints([0] + list(torch.tensor(sizes).cumsum(0)))
    rows = torch.randint(0, n, (m + 2,), generator=g, device="cuda", dtype=torch.int32)
    y = torch.full((m + 2, o), 3.0, device="cuda", dtype=dtype)
    gpu.cnn_fc_grouped_fwd(xq, w, offsets, b, rows=rows, w_scale=ws, x_scale=xs, y_dtype=dtype, y=y)
    check_grouped(y, ref.values(xq, xs, i), wv, offsets, rows, b, False, f"mx4 {dtype}", untouched=3.0)


@pytest.mark.parametrize("kind", ["wide", "mx4"])
@pytest.mark.parametrize("each", [1, 30, 200])
def test_fc_grouped_rows_outside_x(gpu, kind, each):
    """Such a row is one of zeros: its result is the bias, even where rows of x hold NaN."""
    g = gen(8)
    i, o = 128, 80
    x = torch.full((4, i), math.nan, device="cuda")
    x[2] = randn((i,), g)
    w, ws, wv = make_weights(kind, 2, o, i, g, torch.float32)
    b = randn((2, o), g)
    rows = ints(([-1, 4, 2**31 - 1, -2**31, 2] * each)[:each] + [2, -7])
    offsets = ints([0, each, each + 2])
    y = gpu.cnn_fc_grouped_fwd(x, w, offsets, b, rows=rows, w_scale=ws)
    clean = x.clone()
    clean[[0, 1, 3]] = 0
    check_grouped(y, clean, wv, offsets, rows, b, False, kind)
    y = gpu.cnn_fc_grouped_fwd(x, w, offsets, b, True, rows=rows, w_scale=ws)
    check_grouped(y, clean, wv, offsets, rows, b, True, kind)


@pytest.mark.parametrize("each", [2, 100])
def test_fc_grouped_offsets_are_cut_to_the_rows(gpu, each):
    """Offsets past M and below 0 reach no memory outside y; groups that lie inside are right."""
    g = gen(12)
    m = 2 * each
    x = randn((m, 64), g)
    w, _, wv = make_weights("wide", 3, 32, 64, g, torch.float32)
    y = torch.full((m, 32), 9.0, device="cuda")
    gpu.cnn_fc_grouped_fwd(x, w, ints([-5, each, 2**31 - 1, 2**31 - 1]), y=y)
    check_grouped(y, x, wv, ints([0, each, m, m]), None, None, False, "cut")
    y = torch.full((m, 32), 9.0, device="cuda")
    gpu.cnn_fc_grouped_fwd(x, w, ints([0, each, 0, 0]), y=y)          # a group that ends before it begins has no rows
    check_grouped(y, x, wv, ints([0, each, each, each]), None, None, False, "decreasing", untouched=9.0)


def test_fc_grouped_many_groups(gpu):
    """More groups than a wave looks at at once, most of them empty."""
    g = gen(13)
    groups, i, o = 300, 64, 48
    sizes = torch.zeros(groups, dtype=torch.long)
    sizes[[0, 63, 64, 65, 200, 299]] = torch.tensor([3, 1, 70, 2, 1, 5])
    offsets = ints([0] + sizes.cumsum(0).tolist())
    for kind in ("wide", "mx4"):
        w, ws, wv = make_weights(kind, groups, o, i, g, torch.bfloat16)
        x = randn((int(sizes.sum()), i), g, torch.bfloat16)
        y = gpu.cnn_fc_grouped_fwd(x, w, offsets, w_scale=ws)
        check_grouped(y, x, wv, offsets, None, None, False, kind)


@pytest.mark.parametrize("kind", ["wide", "mx4"])
def test_fc_grouped_weights_past_32_bits(gpu, kind):
    """Weights of more than 2^32 bytes (wide) and 2^32 values (mx4): the last group reads its own."""
    g = gen(14)
    i, o = 4096, 4096
    groups = 140 if kind == "wide" else 270
    if kind == "wide":
        w, ws = torch.zeros((groups, o, i), device="cuda", dtype=torch.bfloat16), None
        w[-1] = randn((o, i), g, torch.bfloat16) / 64
        last = w[-1].double()
    else:
        w = torch.zeros((groups, o, i // 2), device="cuda", dtype=torch.uint8)
        ws = torch.full((groups, o, i // 32), 120, device="cuda", dtype=torch.uint8)
        w[-1], ws[-1] = ref.random_mx4((o,), i, g)
        last = ref.values(w[-1], ws[-1], i)
    for each in (2, 60):
        x = randn((2 * each, i), g, torch.bfloat16)
        offsets = ints([0] + [each] * (groups - 1) + [2 * each])
        y = gpu.cnn_fc_grouped_fwd(x, w, offsets, w_scale=ws)
        want, s = ref.product(x[each:], last, None, False)
        ref.assert_product(y[each:], want, s, i, kind)
        assert float(y[:each].abs().max()) == 0


def test_fc_grouped_refuses(gpu):
    g = gen(15)
    x, w, off = randn((6, 64), g), randn((2, 8, 64), g), ints([0, 3, 6])
    with pytest.raises(TypeError):
        gpu.cnn_fc_grouped_fwd(x, w, off.long())
    with pytest.raises(ValueError):
        gpu.cnn_fc_grouped_fwd(x, w, off[:2].contiguous())
    with pytest.raises(ValueError):
        gpu.cnn_fc_grouped_fwd(x, w[..., :32].contiguous(), off)
    with pytest.raises(TypeError):
        gpu.cnn_fc_grouped_fwd(x, w.transpose(1, 2), off)
    with pytest.raises(TypeError):
        gpu.cnn_fc_grouped_fwd(x, w, off.cpu())
    with pytest.raises(gpu.CnnError):
        gpu.cnn_fc_grouped_fwd(x, w.bfloat16(), off)
    with pytest.raises(ValueError):
        gpu.cnn_fc_grouped_fwd(x, w, off, bias=torch.zeros((8,), device="cuda"))
    assert gpu.cnn_fc_grouped_fwd(x[:0], w, ints([0, 0, 0])).shape == (0, 8)


# ---------------------------------------------------------------- routing
def check_route(gpu, logits, k, renorm):
    got = gpu.cnn_route_fwd(logits, k, renormalize=renorm)
    want = ref.route(logits, k, renorm)
    for name, a, b in zip(("expert", "weight", "rows", "offsets", "slot"), got, want):
        if name != "weight":
            assert a.dtype == torch.int32 and torch.equal(a, b), name
    w, r = got[1].double(), want[1]
    # exp of a difference of logits that is exact in fp32 up to 2^-24 of it: with differences below 2^7 the
    # exponent is off by 2^-17 at most; the sums of up to 1024 terms and the quotient add 2^-13 less
    assert float((w - r).abs().max() if w.numel() else 0) <= 2.0 ** -16
    assert bool(((w - r).abs() <= 2.0 ** -16 * r + 1e-30).all())


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("t,e,k", [(1, 1, 1), (1, 8, 2), (16, 128, 4), (63, 7, 7), (64, 64, 8), (65, 64, 8), (100, 65, 1),
                                   (129, 1024, 64), (500, 3, 3), (4097, 60, 6), (8192, 300, 8), (20000, 16, 2)])
def test_route(gpu, dtype, renorm, t, e, k):
    check_route(gpu, 2 * randn((t, e), gen(t + e + k), dtype), k, renorm)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("t,e,k", [(33, 64, 8), (48, 128, 4), (49, 128, 4), (64, 33, 5), (64, 256, 8), (32, 257, 3), (33, 512, 8),
                                   (1, 512, 2), (200, 300, 64), (3000, 511, 8), (64, 1024, 64)])
def test_route_of_more_experts(gpu, dtype, renorm, t, e, k):
    logits = randn((t, e), gen(t + e), dtype)
    logits[::3, ::7] = -math.inf
    logits[1::5, 1::11] = math.nan
    logits[::2, 3::13] = 0.0
    logits[::2, 4::13] = -0.0
    check_route(gpu, logits, k, renorm)


@pytest.mark.parametrize("t", [3, 200])
def test_route_ties(gpu, t):
    """Equal logits go to the lower expert; +0 and -0 are equal."""
    g = gen(21)
    check_route(gpu, torch.randint(0, 3, (t, 200), generator=g, device="cuda").float(), 9, True)
    zeros = torch.zeros((t, 130), device="cuda")
    zeros[:, ::2] = -0.0
    check_route(gpu, zeros, 5, False)


@pytest.mark.parametrize("t", [5, 300])
@pytest.mark.parametrize("renorm", [False, True])
def test_route_masked(gpu, t, renorm):
    """Minus infinity and NaN are never chosen: rows with fewer experts than choices, and with none; the type's
    lowest value is chosen like any other."""
    g = gen(22)
    for dtype in TYPES:
        x = 2 * randn((t, 40), g, dtype)
        keep = torch.randint(0, 41, (t, 1), generator=g, device="cuda")
        x = torch.where(torch.arange(40, device="cuda") < keep, x, -math.inf)
        x[0] = -math.inf
        x[1, ::3] = math.nan
        x[2] = math.nan
        check_route(gpu, x.to(dtype).contiguous(), 6, renorm)
        low = torch.full((t, 40), torch.finfo(dtype).min, device="cuda", dtype=dtype)
        low[:, 7] = -math.inf
        check_route(gpu, low, 3, renorm)


def test_route_plus_infinity_stays_in_range(gpu):
    x = torch.zeros((70, 20), device="cuda")
    x[3, 5] = math.inf
    expert, weight, rows, offsets, slot = gpu.cnn_route_fwd(x, 2)
    assert expert[3].tolist() == [5, 0] and int(offsets[-1]) == 140
    assert bool(torch.isnan(weight[3]).any()) and bool(torch.isfinite(weight[4:]).all())


def test_route_no_tokens(gpu):
    expert, weight, rows, offsets, slot = gpu.cnn_route_fwd(torch.empty((0, 1000), device="cuda"), 4)
    assert expert.shape == (0, 4) and rows.numel() == 0 and offsets.tolist() == [0] * 1001
    with pytest.raises(gpu.CnnError):
        gpu.cnn_route_fwd(torch.zeros((3, 4), device="cuda"), 5)
    with pytest.raises(TypeError):
        gpu.cnn_route_fwd(torch.zeros((4, 3), device="cuda").t(), 2)


# ---------------------------------------------------------------- combining
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,k,d", [(1, 1, 1), (33, 3, 1013), (5, 8, 64), (200, 2, 2048), (3, 64, 7), (1000, 4, 12)])
def test_combine(gpu, dtype, n, k, d):
    g = gen(n + k + d)
    m = n * k
    x = randn((m, d), g, dtype)
    slot = torch.randint(-1, m + 1, (n, k), generator=g, device="cuda", dtype=torch.int32)
    slot[0] = -1
    weight = torch.rand((n, k), generator=g, device="cuda")
    there = (slot >= 0) & (slot < m)
    weight[~there] = math.nan                        # of what is not there, nothing counts
    y = gpu.cnn_combine_fwd(x, slot, weight)
    terms = x[slot.clamp(0, m - 1).long()].double() * weight.double().unsqueeze(-1)
    terms = torch.where(there.unsqueeze(-1), terms, 0.0)
    want, s = terms.sum(1), terms.abs().sum(1)
    ref.assert_product(y, want, s, k, f"{dtype} {n}x{k}x{d}")
    assert float(y[0].abs().max()) == 0


def test_combine_empty_and_refused(gpu):
    x, slot, weight = torch.ones((4, 8), device="cuda"), ints([[0, 1]]), torch.ones((1, 2), device="cuda")
    assert gpu.cnn_combine_fwd(x, slot[:0], weight[:0]).shape == (0, 8)
    assert float(gpu.cnn_combine_fwd(x[:0], slot, weight).abs().max()) == 0    # no rows: every slot is outside
    with pytest.raises(ValueError):
        gpu.cnn_combine_fwd(x, slot, weight[:, :1].contiguous())
    with pytest.raises(TypeError):
        gpu.cnn_combine_fwd(x, slot.long(), weight)
    with pytest.raises(TypeError):
        gpu.cnn_combine_fwd(x, slot, weight.double())


# ---------------------------------------------------------------- together
class Block:
    """A served block: k of E experts, two layers each."""

    def __init__(self, gpu, kind, dtype, t, e, k, d, h, seed):
        g = gen(seed)
        self.gpu, self.k, self.dtype = gpu, k, dtype
        self.x = randn((t, d), g, dtype)
        self.logits = 1.5 * randn((t, e), g)
        self.w1, self.s1, self.v1 = make_weights(kind, e, h, d, g, dtype)
        self.w2, self.s2, self.v2 = make_weights(kind, e, d, h, g, dtype)
        self.b1, self.b2 = 0.1 * randn((e, h), g), 0.1 * randn((e, d), g)

    def __call__(self, x=None, logits=None, stream=None):
        gpu, x = self.gpu, self.x if x is None else x
        _, weight, rows, offsets, slot = gpu.cnn_route_fwd(self.logits if logits is None else logits, self.k,
                                                           renormalize=True, stream=stream)
        h = gpu.cnn_fc_grouped_fwd(x, self.w1, offsets, self.b1, True, rows=rows, w_scale=self.s1, stream=stream)
        y = gpu.cnn_fc_grouped_fwd(h, self.w2, offsets, self.b2, w_scale=self.s2, stream=stream)
        return gpu.cnn_combine_fwd(y, slot, weight, stream=stream)

    def reference(self):
        """The block in float64, every token through all of its experts, and a bound for the result.

        h is rounded to the type (eps/2) with the error of its sums; y carries it through |w2|, adds its own; the
        combination adds k + 2 steps and a rounding.  Weights are off by 2^-16 at most (check_route)."""
        expert, weight, *_ = ref.route(self.logits, self.k, True)
        half = torch.finfo(self.dtype).eps / 2
        out = torch.zeros((self.x.shape[0], self.v2.shape[1]), dtype=torch.float64, device="cuda")
        off = torch.zeros_like(out)
        for j in range(self.k):
            for e in range(self.v1.shape[0]):
                at = (expert[:, j] == e).nonzero().flatten()
                if not at.numel():
                    continue
                n1, n2 = self.v1.shape[2], self.v2.shape[2]
                h, s = ref.product(self.x[at], self.v1[e], self.b1[e], True)
                dh = half * h + (n1 + 2) * 2.0 ** -23 * s
                y, s = ref.product(h, self.v2[e], self.b2[e], False)
                dy = dh @ self.v2[e].abs().T
                dy = dy + (1 + half) * (n2 + 2) * 2.0 ** -23 * (s + dy) + half * (y.abs() + dy)
                wt = weight[at, j].unsqueeze(1)
                out[at] += wt * y
                off[at] += wt * (dy + (2.0 ** -16 + (self.k + 2) * 2.0 ** -23) * (y.abs() + dy))
        return out, off + half * (out.abs() + off) + 1e-7


def assert_block(y, want, off, what):
    worst = float(((y.double() - want).abs() / off).max())
    assert worst <= 1, f"{what}: {worst:.3g} of its bound"


@pytest.mark.parametrize("kind", ["wide", "mx4"])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("t,e,k,d,h", [(1, 8, 2, 256, 512), (9, 16, 4, 96, 100), (200, 5, 2, 130, 190), (700, 8, 2, 256, 384)])
def test_block(gpu, kind, dtype, t, e, k, d, h):
    block = Block(gpu, kind, dtype, t, e, k, d, h, t)
    want, off = block.reference()
    assert_block(block(), want, off, f"{kind} {dtype}")


@pytest.mark.parametrize("t", [4, 300])
def test_block_masked_tokens(gpu, t):
    """Padded tokens (logits of minus infinity) have no expert: their results are zero, the others' stay."""
    block = Block(gpu, "mx4", torch.bfloat16, t, 8, 2, 128, 256, 31)
    whole = block()
    pad = torch.arange(t, device="cuda") % 3 == 1
    logits = block.logits.masked_fill(pad.unsqueeze(1), -math.inf)
    y = block(logits=logits)
    assert float(y[pad].abs().max()) == 0
    # with fewer rows an expert may take another kernel, whose sums run in another order
    want, off = block.reference()
    assert_block(y[~pad], want[~pad], off[~pad], "unpadded")
    assert_block(whole, want, off, "whole")


@pytest.mark.parametrize("kind", ["wide", "mx4"])
@pytest.mark.parametrize("t", [3, 150])
def test_block_captured(gpu, kind, t):
    """Captured and replayed with new inputs in the same buffers, with eager work of its own between; two graphs
    of it do not share anything."""
    block = Block(gpu, kind, torch.bfloat16, t, 8, 2, 128, 256, 41)
    block()
    torch.cuda.synchronize()
    x, logits = block.x.clone(), block.logits.clone()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = block(x, logits)
        graphs.append((g, y))
    for i in range(3):
        r = gen(50 + i)
        x.copy_(randn(x.shape, r, x.dtype))
        logits.copy_(randn(logits.shape, r))
        eager = block(x, logits)
        for g, y in graphs:
            y.fill_(math.nan)
        for g, _ in graphs:
            g.replay()
        between = block()
        torch.cuda.synchronize()
        for _, y in graphs:
            assert torch.equal(y, eager), i
        assert bool(torch.isfinite(between).all())


@pytest.mark.parametrize("t", [5, 400])
def test_block_on_another_stream(gpu, t):
    """Two passes at once on streams of their own, given as an argument and as the current stream."""
    one = Block(gpu, "mx4", torch.bfloat16, t, 8, 2, 128, 256, 61)
    two = Block(gpu, "wide", torch.float32, t, 8, 2, 128, 256, 62)
    want = one(), two()
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        got_one = one(stream=a)
        with torch.cuda.stream(b):
            got_two = two()
        raw = two(stream=a.cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(got_one, want[0]) and torch.equal(got_two, want[1]) and torch.equal(raw, want[1])
