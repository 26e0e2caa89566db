"""Microscaled 4-bit values (GPU): conversion both ways and the fully connected
layer on them, against references in 64 bits (``experts_ref``)."""
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


def randn(shape, g, dtype=torch.float32, spread=0.0):
    x = torch.randn(shape, generator=g, device="cuda")
    if spread:
        x = x * torch.exp(spread * torch.randn(shape[-1:], generator=g, device="cuda"))
    return x.to(dtype)


# ---------------------------------------------------------------- conversion
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 33), (7, 31), (5, 64), (64, 4096), (2, 8200), (1000, 7),
                                       (4097, 96)])
def test_quantize(gpu, dtype, rows, cols):
    x = randn((rows, cols), gen(rows + cols), dtype, spread=2.0)
    q, s = gpu.cnn_mx4_quantize(x)
    rq, rs = ref.quantize(x)
    assert torch.equal(s, rs)
    assert torch.equal(q, rq)
    y = gpu.cnn_mx4_dequantize(q, s, cols, dtype=dtype)
    assert torch.equal(y.double(), ref.values(rq, rs, cols).to(dtype).double())


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_quantize_midpoints_and_extremes(gpu, dtype):
    """Every multiple of 1/16 below 8, both signs, at several scales; zeros, the type's largest and smallest
    values, infinities and NaN."""
    steps = torch.arange(0, 128, device="cuda", dtype=torch.float64) / 16
    steps = torch.stack([steps, -steps], 1).reshape(8, 32)
    steps[:, 0] = 4.0                                # fixes the scale of the block
    info = torch.finfo(dtype)
    rows = [steps.reshape(1, -1) * 2.0 ** e for e in (0, -7, 5)]
    edge = torch.zeros((8, 32), device="cuda", dtype=torch.float64)
    edge[1, 5] = info.max
    edge[2] = -info.max
    edge[3, 31] = info.smallest_normal
    edge[4, 0] = info.smallest_normal * info.eps     # the smallest subnormal
    edge[5, 9], edge[5, 10] = math.inf, 1.0
    edge[6, 1] = -math.inf
    edge[7, 30], edge[7, 2] = math.nan, 3.0
    x = torch.cat(rows + [edge.reshape(1, -1)]).to(dtype).contiguous()
    q, s = gpu.cnn_mx4_quantize(x)
    rq, rs = ref.quantize(x)
    assert torch.equal(s, rs) and torch.equal(q, rq)
    y = gpu.cnn_mx4_dequantize(q, s, 256, dtype=torch.float32)
    want = ref.values(rq, rs, 256)
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    assert torch.equal(y.nan_to_num().double(), want.nan_to_num().float().double())
    assert bool(torch.isnan(y[3].reshape(8, 32)[5:]).all()) and not bool(torch.isnan(y[3].reshape(8, 32)[:5]).any())


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_dequantize_every_code_and_scale(gpu, dtype):
    q = torch.arange(16, dtype=torch.uint8, device="cuda") * 17
    q = q.repeat(256, 1)                             # a block holds every code twice
    s = torch.arange(256, dtype=torch.uint8, device="cuda").reshape(256, 1)
    y = gpu.cnn_mx4_dequantize(q, s, dtype=dtype)
    want = ref.values(q, s, 32).to(dtype)
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    assert torch.equal(y.nan_to_num(7.0), want.nan_to_num(7.0))


def test_conversion_of_views_and_leading_dimensions(gpu):
    """Rows that start at any element (an odd width, a row offset), three dimensions, outputs given."""
    base = randn((5, 77), gen(5), torch.bfloat16)
    x = base[1:]
    q, s = gpu.cnn_mx4_quantize(x)
    rq, rs = ref.quantize(x)
    assert torch.equal(q, rq) and torch.equal(s, rs)
    x3 = randn((3, 4, 50), gen(6))
    q, s = gpu.cnn_mx4_quantize(x3)
    assert q.shape == (3, 4, 32) and s.shape == (3, 4, 2)
    rq, rs = ref.quantize(x3.reshape(12, 50))
    assert torch.equal(q.reshape(12, -1), rq) and torch.equal(s.reshape(12, -1), rs)
    out = torch.full((3, 4, 50), -1.0, device="cuda", dtype=torch.float16)
    assert gpu.cnn_mx4_dequantize(q, s, 50, y=out) is out
    assert torch.equal(out.reshape(12, 50).double(), ref.values(rq, rs, 50).half().double())
    q, s = gpu.cnn_mx4_quantize(torch.empty((0, 40), device="cuda"))
    assert q.shape == (0, 32) and gpu.cnn_mx4_dequantize(q, s, 40).shape == (0, 40)
    with pytest.raises(TypeError):
        gpu.cnn_mx4_quantize(base.t())
    with pytest.raises(TypeError):
        gpu.cnn_mx4_quantize(base.double())
    with pytest.raises(ValueError):
        gpu.cnn_mx4_dequantize(rq, rs, 32)      # one block would hold them
    with pytest.raises(ValueError):
        gpu.cnn_mx4_quantize(x3, q=torch.empty((3, 4, 16), dtype=torch.uint8, device="cuda"))


# ---------------------------------------------------------------- fully connected
SHAPES = [(1, 1, 1), (1, 32, 16), (1, 33, 1), (2, 7, 5), (3, 64, 17), (5, 100, 130), (16, 512, 1000), (17, 2048, 33),
          (33, 610, 188), (48, 160, 40), (64, 129, 256), (1, 4096, 1000), (130, 1024, 257), (300, 96, 700), (513, 384, 512),
          (1030, 513, 129)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,i,o", SHAPES)
def test_fc_mx4(gpu, dtype, n, i, o):
    g = gen(n + i + o)
    x = randn((n, i), g, dtype, spread=0.5)
    w, ws = ref.random_mx4((o,), i, g)
    b = 0.1 * randn((o,), g)
    wv = ref.values(w, ws, i)
    for bias, relu in ((b, False), (None, False), (b, True)):
        y = gpu.cnn_fc_mx4_fwd(x, w, ws, bias, relu)
        assert y.dtype == dtype
        want, s = ref.product(x, wv, bias, relu)
        ref.assert_product(y, want, s, i, f"{dtype} {n}x{i}x{o} bias {bias is not None} relu {relu}")


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,i,o", SHAPES)
def test_fc_mx4_of_mx4_inputs(gpu, dtype, n, i, o):
    g = gen(n + i + o + 1)
    xq, xs = gpu.cnn_mx4_quantize(randn((n, i), g, dtype, spread=0.5))
    w, ws = ref.random_mx4((o,), i, g)
    b = 0.1 * randn((o,), g)
    y = gpu.cnn_fc_mx4_fwd(xq, w, ws, b, x_scale=xs, y_dtype=dtype)
    assert y.dtype == dtype
    want, s = ref.product(ref.values(xq, xs, i), ref.values(w, ws, i), b, False)
    ref.assert_product(y, want, s, i, f"mx4 to {dtype} {n}x{i}x{o}")


def off_by_one(x):
    """The same tensor at an address that is aligned to its elements only."""
    flat = torch.empty(x.numel() + 1, dtype=x.dtype, device=x.device)
    flat[1:] = x.reshape(-1)
    return flat[1:].view(x.shape)


# enough rows and outputs for the larger tiles, with and without a tail that is split along the reduction
LARGE = [(2100, 304, 4100), (4200, 136, 4100), (4200, 1032, 4100), (1500, 2048, 2100)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,i,o", LARGE)
def test_fc_mx4_large(gpu, dtype, n, i, o):
    g = gen(n + i + o)
    x = randn((n, i), g, dtype, spread=0.5)
    w, ws = ref.random_mx4((o,), i, g)
    b = 0.1 * randn((o,), g)
    wv = ref.values(w, ws, i)
    want, s = ref.product(x, wv, b, True)
    ref.assert_product(gpu.cnn_fc_mx4_fwd(x, w, ws, b, True), want, s, i, f"{dtype} {n}x{i}x{o}")
    ref.assert_product(gpu.cnn_fc_mx4_fwd(off_by_one(x), w, ws, b, True), want, s, i, f"{dtype} {n}x{i}x{o} unaligned")
    xq, xs = gpu.cnn_mx4_quantize(x)
    want, s = ref.product(ref.values(xq, xs, i), wv, b, False)
    ref.assert_product(gpu.cnn_fc_mx4_fwd(xq, w, ws, b, x_scale=xs, y_dtype=dtype), want, s, i, f"mx4 to {dtype} {n}x{i}x{o}")


@pytest.mark.parametrize("n,i,o", [(4000, 304, 4000), (3800, 136, 7900), (8100, 1032, 8300)])
def test_fc_mx4_largest(gpu, n, i, o):
    """The largest tiles: one whole round of them, a last one that is nearly whole, a tail that is split."""
    g = gen(n + i + o)
    x = randn((n, i), g, torch.bfloat16, spread=0.5)
    w, ws = ref.random_mx4((o,), i, g)
    b = 0.1 * randn((o,), g)
    want, s = ref.product(x, ref.values(w, ws, i), b, True)
    y = gpu.cnn_fc_mx4_fwd(x, w, ws, b, True)
    ref.assert_product(y, want, s, i, f"{n}x{i}x{o}")
    assert torch.equal(gpu.cnn_fc_mx4_fwd(x, w, ws, b, True), y)
    ref.assert_product(gpu.cnn_fc_mx4_fwd(off_by_one(x), w, ws, b, True), want, s, i, f"{n}x{i}x{o} unaligned")


@pytest.mark.parametrize("n", [1, 40, 300])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_fc_mx4_is_the_same_from_call_to_call(gpu, n, dtype):
    g = gen(n)
    x = randn((n, 1111), g, dtype)
    w, ws = ref.random_mx4((333,), 1111, g)
    first = gpu.cnn_fc_mx4_fwd(x, w, ws)
    for _ in range(3):
        assert torch.equal(gpu.cnn_fc_mx4_fwd(x, w, ws), first)


@pytest.mark.parametrize("n", [1, 20, 200])
def test_fc_mx4_small_parts_of_fp32_inputs(gpu, n):
    """fp32 inputs keep all 24 bits: x = 1 + 2^-23 against weights whose sum cancels the ones."""
    i, o = 256, 64
    x = torch.full((n, i), 1.0 + 2.0 ** -23, device="cuda")
    x[:, 1::2] = 1.0
    q = torch.full((o, i // 2), 0x2 | (0xA << 4), dtype=torch.uint8, device="cuda")   # +1, -1, +1, ...
    s = torch.full((o, i // 32), 127, dtype=torch.uint8, device="cuda")
    y = gpu.cnn_fc_mx4_fwd(x, q, s)
    # partial sums stay within 32 ones, in which 2^-23 is an exact multiple of nothing lost: the sum is
    # 128 times 2^-23 = 2^-16, and no partial sum of it above 32 + 2^-16 is cut below 2^-19
    assert float((y.double() - 2.0 ** -16).abs().max()) <= 256 * 2.0 ** -19


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n", [1, 17, 150])
def test_fc_mx4_nan_and_infinity(gpu, dtype, n):
    """An infinite or NaN input reaches its own row and no other; a NaN block of the weights its own column.
    Infinity times a nonzero weight is infinity."""
    g = gen(9)
    i, o = 300, 70
    x = randn((n, i), g, dtype)
    w, ws = ref.random_mx4((o,), i, g)
    w[:, 5] = 0x22                                   # columns 10 and 11: weights of +1
    good = gpu.cnn_fc_mx4_fwd(x, w, ws)
    ws2 = ws.clone()
    ws2[33, 9] = 255                                 # the last, partial block of a column
    y = gpu.cnn_fc_mx4_fwd(x, w, ws2)
    assert bool(torch.isnan(y[:, 33]).all())
    keep = torch.arange(o, device="cuda") != 33
    assert torch.equal(y[:, keep], good[:, keep])
    r = n // 2
    for bad in (math.inf, -math.inf, math.nan):
        x2 = x.clone()
        x2[r, 10] = bad
        y = gpu.cnn_fc_mx4_fwd(x2, w, ws)
        others = torch.arange(n, device="cuda") != r
        assert torch.equal(y[others], good[others])
        if math.isnan(bad):
            assert bool(torch.isnan(y[r]).all())
        else:
            assert bool((y[r] == bad).all()), y[r]
    largest = torch.zeros((n, i), device="cuda", dtype=dtype)
    largest[:, 10] = torch.finfo(dtype).max
    half = torch.full_like(w, 0)
    half[:, 5] = 0x01                                # column 10: 0.5
    s = torch.full_like(ws, 127)
    y = gpu.cnn_fc_mx4_fwd(largest, half, s)
    assert bool((y == torch.finfo(dtype).max / 2).all())


def test_fc_mx4_shapes_strides_and_empty(gpu):
    g = gen(3)
    w, ws = ref.random_mx4((40,), 72, g)
    x = randn((6, 2, 6, 6), g)                       # read flattened
    want, s = ref.product(x.reshape(6, 72), ref.values(w, ws, 72), None, False)
    ref.assert_product(gpu.cnn_fc_mx4_fwd(x, w, ws), want, s, 72, "flattened")
    x = randn((7, 72), g, torch.bfloat16)[1:]        # a row offset
    want, s = ref.product(x, ref.values(w, ws, 72), None, False)
    out = torch.empty((6, 40), device="cuda", dtype=torch.bfloat16)
    assert gpu.cnn_fc_mx4_fwd(x, w, ws, y=out) is out
    ref.assert_product(out, want, s, 72, "offset rows")
    odd = randn((7, 71), g, torch.bfloat16)[1:]      # rows on odd half-words
    w1, ws1 = ref.random_mx4((40,), 71, g)
    want, s = ref.product(odd, ref.values(w1, ws1, 71), None, False)
    ref.assert_product(gpu.cnn_fc_mx4_fwd(odd, w1, ws1), want, s, 71, "odd rows")
    assert gpu.cnn_fc_mx4_fwd(x[:0], w, ws).shape == (0, 40)
    assert gpu.cnn_fc_mx4_fwd(torch.empty((0, 2, 6, 6), device="cuda"), w, ws).shape == (0, 40)
    with pytest.raises(TypeError):
        gpu.cnn_fc_mx4_fwd(randn((72, 6), g).t(), w, ws)
    with pytest.raises(ValueError):
        gpu.cnn_fc_mx4_fwd(randn((6, 97), g), w, ws)
    with pytest.raises(ValueError):
        gpu.cnn_fc_mx4_fwd(randn((6, 64), g), w, ws)
    with pytest.raises(TypeError):
        gpu.cnn_fc_mx4_fwd(randn((6, 72), g), w, ws, bias=torch.zeros(40, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        gpu.cnn_fc_mx4_fwd(randn((6, 72), g), w, ws, bias=torch.zeros(39, device="cuda"))
    with pytest.raises(TypeError):
        gpu.cnn_fc_mx4_fwd(randn((6, 72), g), w, ws, y=torch.empty((6, 40), device="cuda", dtype=torch.float16))


def test_sizes_past_the_limit_are_refused(gpu):
    x = torch.empty(2**31 + 64, dtype=torch.bfloat16, device="cuda").reshape(-1, 32)
    with pytest.raises(gpu.CnnError):
        gpu.cnn_mx4_quantize(x)
    with pytest.raises(gpu.CnnError):
        gpu.cnn_combine_fwd(x, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.zeros((1, 1), device="cuda"))


def test_fc_mx4_rows_past_32_bits(gpu):
    """Inputs of more than 4 GiB: the last rows are read where they are."""
    n, i, o = 300_000, 4096, 16
    x = torch.zeros((n, i), device="cuda")
    g = gen(4)
    x[-3:] = randn((3, i), g)
    x[100] = randn((i,), g)
    w, ws = ref.random_mx4((o,), i, g)
    y = gpu.cnn_fc_mx4_fwd(x, w, ws)
    at = [100, n - 3, n - 2, n - 1]
    want, s = ref.product(x[at], ref.values(w, ws, i), None, False)
    ref.assert_product(y[at], want, s, i, "far rows")
    assert float(y[101:n - 3].abs().max()) == 0
