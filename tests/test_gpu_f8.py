"""8-bit floats with a scale for each block of 128 (GPU): conversion both ways
and the fully connected layer on them, against references in 64 bits
(``head_ref``)."""
import math

import pytest
import torch

import head_ref as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
IDS = ["f32", "bf16", "f16"]
F8 = ref.F8


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
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 129), (7, 127), (129, 64), (64, 4096), (2, 8200), (1000, 7),
                                       (300, 389), (257, 256)])
def test_quantize(gpu, dtype, block_rows, rows, cols):
    x = randn((rows, cols), gen(rows + cols), dtype, spread=2.0)
    q, s = gpu.cnn_f8_quantize(x, block_rows)
    rq, rs = ref.quantize(x, block_rows)
    assert torch.equal(s, rs)
    assert torch.equal(q.double(), rq)
    for out in TYPES:
        y = gpu.cnn_f8_dequantize(q, s, block_rows, dtype=out)
        want = (rq * ref.spread(rs, rows, cols, block_rows)).float().to(out)
        assert torch.equal(y, want)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_quantize_midpoints_and_extremes(gpu, dtype):
    """Codes, midpoints between them and their neighbours, both signs; zeros, the type's largest and smallest values,
    infinities and NaN."""
    codes = torch.arange(0, 127, device="cuda", dtype=torch.uint8).view(F8).double()
    mid = (codes[1:] + codes[:-1]) / 2
    v = torch.cat([codes, mid, mid * (1 + 2.0 ** -10), mid * (1 - 2.0 ** -10)])
    v = torch.cat([v, -v])
    v = torch.nn.functional.pad(v, (0, -len(v) % 127)).reshape(-1, 127)
    v = torch.cat([torch.full_like(v[:, :1], 448.0), v], 1)       # fixes the scale at 1
    info = torch.finfo(dtype)
    edge = torch.zeros((8, 128), device="cuda", dtype=torch.float64)
    edge[1, 5] = info.max
    edge[2] = -info.max
    edge[3, 31] = info.smallest_normal
    edge[4, 0] = info.smallest_normal * info.eps     # the smallest subnormal
    edge[5, 9], edge[5, 10] = math.inf, 1.0
    edge[6, 1] = -math.inf
    edge[7, 30], edge[7, 2] = math.nan, 3.0
    x = torch.cat([v, edge]).to(dtype).contiguous()
    for br in (1, 128):
        for part in (x, x[len(v):].contiguous(), x[len(v):-3].contiguous()):
            q, s = gpu.cnn_f8_quantize(part, br)
            rq, rs = ref.quantize(part, br)
            assert torch.equal(s.isnan(), rs.isnan()) and torch.equal(s.nan_to_num(-1), rs.nan_to_num(-1))
            assert torch.equal(q.double(), rq)
    y = gpu.cnn_f8_dequantize(*gpu.cnn_f8_quantize(x))
    assert bool(y[-1].isnan().all()) and bool(y[-2].isnan().all()) and not bool(y[-4].isnan().any())


def test_quantize_leading_dimensions_and_places(gpu):
    x = randn((3, 5, 200), gen(1), torch.bfloat16)
    q, s = gpu.cnn_f8_quantize(x)
    assert q.shape == (3, 5, 200) and s.shape == (3, 5, 2)
    rq, rs = ref.quantize(x.reshape(15, 200))
    assert torch.equal(q.double().reshape(15, 200), rq) and torch.equal(s.reshape(15, 2), rs)
    assert gpu.cnn_f8_dequantize(q, s, dtype=torch.float16).shape == x.shape
    # an 8-bit tensor may begin at any byte
    room = torch.empty(15 * 200 + 3, dtype=torch.uint8, device="cuda")
    at = room[3:].view(F8).view(15, 200)
    q2, _ = gpu.cnn_f8_quantize(x.reshape(15, 200), q=at)
    assert q2.data_ptr() == at.data_ptr() and torch.equal(at.double(), rq)
    assert torch.equal(gpu.cnn_f8_dequantize(at, s.reshape(15, 2)), (rq * ref.spread(rs, 15, 200, 1)).float())
    e = torch.empty((0, 200), device="cuda")
    q, s = gpu.cnn_f8_quantize(e)
    assert q.shape == (0, 200) and s.shape == (0, 2) and gpu.cnn_f8_dequantize(q, s).shape == (0, 200)


def test_conversions_refuse(gpu):
    x = torch.ones((4, 256), device="cuda")
    q, s = gpu.cnn_f8_quantize(x)
    for call, error in [
        (lambda: gpu.cnn_f8_quantize(x.double()), TypeError),
        (lambda: gpu.cnn_f8_quantize(x.cpu()), TypeError),
        (lambda: gpu.cnn_f8_quantize(x.T), TypeError),
        (lambda: gpu.cnn_f8_quantize(x[0]), ValueError),
        (lambda: gpu.cnn_f8_quantize(x, 64), ValueError),
        (lambda: gpu.cnn_f8_quantize(x.reshape(2, 2, 256), 128), ValueError),
        (lambda: gpu.cnn_f8_quantize(x, q=q.view(torch.uint8)), TypeError),
        (lambda: gpu.cnn_f8_quantize(x, scale=s[:3].contiguous()), ValueError),
        (lambda: gpu.cnn_f8_dequantize(q, s[:, :1].contiguous()), ValueError),
        (lambda: gpu.cnn_f8_dequantize(q, s, 128), ValueError),
        (lambda: gpu.cnn_f8_dequantize(q.view(torch.uint8), s), TypeError),
        (lambda: gpu.cnn_f8_dequantize(q, s.double()), TypeError),
        (lambda: gpu.cnn_f8_dequantize(q, s, dtype=torch.float64), TypeError),
        (lambda: gpu.cnn_f8_quantize(torch.ones((4, 0), device="cuda")), gpu.CnnError),
    ]:
        with pytest.raises(error):
            call()


# ---------------------------------------------------------------- the product
def operands(n, i, o, seed, spread=0.5):
    g = gen(seed)
    x, w = ref.random_f8((n, i), g), ref.random_f8((o, i), g)
    nb = ref.blocks_of(i)
    xs = torch.exp(spread * randn((n, nb), g)) / 100
    ws = torch.exp(spread * randn((ref.blocks_of(o), nb), g)) / (100 * math.sqrt(i))
    return x, xs, w, ws, 0.1 * randn((o,), g)


def check(gpu, n, i, o, dtype, bias, relu, seed=None):
    x, xs, w, ws, b = operands(n, i, o, n + i + o if seed is None else seed)
    b = b if bias else None
    y = gpu.cnn_fc_f8_fwd(x, xs, w, ws, b, relu, y_dtype=dtype)
    want, s = ref.product(x, xs, w, ws, b, relu)
    ref.assert_product(y, want, s, i, f"{n}x{i}x{o} {dtype}")
    return y


SIZES = [(1, 1, 1), (1, 128, 16), (2, 127, 17), (3, 129, 130), (1, 4096, 512), (5, 1000, 333), (16, 256, 1000), (17, 384, 99),
         (31, 2000, 128), (33, 640, 257), (64, 1024, 1000), (65, 4096, 131), (77, 1013, 610), (128, 512, 384),
         (200, 3000, 200), (255, 130, 511), (257, 1152, 513), (600, 264, 70), (1025, 384, 640), (1, 9216, 10), (300, 16, 4096)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,i,o", SIZES)
def test_product(gpu, n, i, o, dtype):
    check(gpu, n, i, o, dtype, bias=True, relu=(n + o) % 2 == 0)


@pytest.mark.parametrize("n,i,o", [(1, 300, 50), (64, 512, 256), (260, 1024, 260)])
def test_product_without_bias(gpu, n, i, o):
    check(gpu, n, i, o, torch.float32, bias=False, relu=False)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_product_adds_in_32_bits(gpu, dtype):
    """Sums whose terms cancel but for one in 2^16: 64 blocks of products of 2^16 and -2^16, and one of 1."""
    for n in (1, 40, 300):
        i, o = 128 * 65, 64
        x = torch.zeros((n, i), device="cuda")
        w = torch.zeros((o, i), device="cuda")
        for k in range(64):
            x[:, 128 * k + k] = 256.0
            w[:, 128 * k + k] = 256.0 if k % 2 else -256.0
        x[:, -1], w[:, -1] = 1.0, 1.0
        one = torch.ones((n, 65), device="cuda")
        y = gpu.cnn_fc_f8_fwd(x.to(F8), one, w.to(F8), torch.ones((1, 65), device="cuda"), y_dtype=dtype)
        assert bool((y == 1.0).all())


def test_product_to_fp32_is_exact_within_a_block(gpu):
    """Products of 2^16, -2^16 and 1 beside each other."""
    for n in (1, 40, 300):
        i, o = 256, 200
        x = torch.zeros((n, i), device="cuda")
        w = torch.zeros((o, i), device="cuda")
        for k in range(0, 240, 3):
            x[:, k], x[:, k + 1], x[:, k + 2] = 256.0, 256.0, 1.0
            w[:, k], w[:, k + 1], w[:, k + 2] = 256.0, -256.0, 1.0
        y = gpu.cnn_fc_f8_fwd(x.to(F8), torch.ones((n, 2), device="cuda"), w.to(F8), torch.ones((2, 2), device="cuda"))
        assert bool((y == 80.0).all())


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_product_blocks_do_not_mix(gpu, dtype):
    """Scales from 2^-60 to 2^60 by the block: every block's own scale counts, in inputs and in weights."""
    for n, o in ((1, 256), (70, 300), (300, 300)):
        i = 640
        x, _, w, _, _ = operands(n, i, o, 5)
        xs = torch.exp2(torch.arange(5, device="cuda", dtype=torch.float32) * 30 - 60).repeat(n, 1)
        xs = (xs * (1 + torch.arange(n, device="cuda").float()[:, None] / n)).contiguous()
        ws = torch.exp2(60 - torch.arange(5, device="cuda", dtype=torch.float32) * 30).repeat(ref.blocks_of(o), 1)
        ws = (ws * (1 + torch.arange(len(ws), device="cuda").float()[:, None])).contiguous()
        xs /= 1024 * 128
        y = gpu.cnn_fc_f8_fwd(x, xs, w, ws, y_dtype=dtype)
        want, s = ref.product(x, xs, w, ws, None, False)
        ref.assert_product(y, want, s, i, f"{n}x{o}")


def test_product_nan_and_its_rows(gpu):
    """NaN in a scale or a value reaches the sums it is part of, and no others."""
    for n, i, o in ((1, 256, 200), (20, 300, 140), (300, 512, 300)):
        x, xs, w, ws, b = operands(n, i, o, 7)
        clean = gpu.cnn_fc_f8_fwd(x, xs, w, ws, b)
        xs2 = xs.clone()
        xs2[n // 2, 1] = math.nan
        y = gpu.cnn_fc_f8_fwd(x, xs2, w, ws, b)
        bad = torch.zeros((n, o), dtype=torch.bool, device="cuda")
        bad[n // 2] = True
        assert torch.equal(y.isnan(), bad) and torch.equal(y[~bad], clean[~bad])
        w2 = w.clone()
        w2.view(torch.uint8)[o - 1, i - 1] = 0x7f
        y = gpu.cnn_fc_f8_fwd(x, xs, w2, ws, b)
        bad[:] = False
        bad[:, o - 1] = True
        assert torch.equal(y.isnan(), bad) and torch.equal(y[~bad], clean[~bad])
        ws2 = ws.clone()
        ws2[-1, 0] = math.inf
        y = gpu.cnn_fc_f8_fwd(x, xs, w, ws2, b)
        bad[:] = False
        bad[:, (o - 1) // 128 * 128:] = True
        assert not bool(y[bad].isfinite().any()) and torch.equal(y[~bad], clean[~bad])
        # ReLU makes NaN 0
        y = gpu.cnn_fc_f8_fwd(x, xs2, w, ws, b, True)
        assert float(y[n // 2].abs().max()) == 0


@pytest.mark.parametrize("n,o", [(3, 50), (20, 33), (70, 300), (2, 8300), (90, 900)])
def test_product_ends_inside_a_block(gpu, n, o):
    """Few tokens: a workgroup's waves share the blocks, the last of which is not whole; waves may have none."""
    for blocks in (*range(1, 35), 63, 70):
        for dtype, i in ((torch.float32, 128 * blocks - 7), (torch.bfloat16, 128 * blocks - 120)):
            check(gpu, n, i, o, dtype, bias=True, relu=False)


@pytest.mark.parametrize("shift", [1, 4, 8])
def test_product_at_any_byte(gpu, shift):
    for n, i, o in ((2, 256, 64), (40, 512, 130), (260, 384, 257)):
        x, xs, w, ws, b = operands(n, i, o, 9)
        want = gpu.cnn_fc_f8_fwd(x, xs, w, ws, b)

        def moved(t):
            room = torch.zeros(t.numel() + 16, dtype=torch.uint8, device="cuda")
            room[:] = 0x7f                                  # NaN on both sides
            at = room[shift:shift + t.numel()]
            at.copy_(t.view(torch.uint8).flatten())
            return at.view(F8).view(t.shape)
        got = gpu.cnn_fc_f8_fwd(moved(x), xs, moved(w), ws, b)
        s = ref.product(x, xs, w, ws, b, False)
        ref.assert_product(got, s[0], s[1], i, "moved")
        assert float((got - want).abs().max()) <= float(s[1].max()) * ref.steps(i) * 2.0 ** -22


def test_product_writes_its_own_rows_only(gpu):
    for n, i, o in ((3, 200, 37), (33, 256, 130), (258, 384, 259)):
        x, xs, w, ws, b = operands(n, i, o, 11)
        room = torch.full((n * o + 64,), 7.0, device="cuda")
        y = room[32:32 + n * o].view(n, o)
        got = gpu.cnn_fc_f8_fwd(x, xs, w, ws, b, y=y)
        assert got.data_ptr() == y.data_ptr()
        assert bool((room[:32] == 7).all()) and bool((room[32 + n * o:] == 7).all())
        assert torch.equal(y, gpu.cnn_fc_f8_fwd(x, xs, w, ws, b))


def test_product_is_the_same_every_time(gpu):
    for n, i, o in ((1, 4096, 1000), (48, 9216, 512), (300, 2048, 600)):
        x, xs, w, ws, b = operands(n, i, o, 13)
        y = gpu.cnn_fc_f8_fwd(x, xs, w, ws, b)
        for _ in range(3):
            assert torch.equal(y, gpu.cnn_fc_f8_fwd(x, xs, w, ws, b))


def test_product_refuses_and_empty(gpu):
    x, xs, w, ws, b = operands(4, 256, 130, 1)
    assert gpu.cnn_fc_f8_fwd(x[:0], xs[:0], w, ws, b).shape == (0, 130)
    for call, error in [
        (lambda: gpu.cnn_fc_f8_fwd(x.float(), xs, w, ws), TypeError),
        (lambda: gpu.cnn_fc_f8_fwd(x, xs, w.view(torch.uint8), ws), TypeError),
        (lambda: gpu.cnn_fc_f8_fwd(x, xs[:, :1].contiguous(), w, ws), ValueError),
        (lambda: gpu.cnn_fc_f8_fwd(x, xs.T, w, ws), TypeError),
        (lambda: gpu.cnn_fc_f8_fwd(x, xs, w, ws[:1]), ValueError),
        (lambda: gpu.cnn_fc_f8_fwd(x, xs, w, ws.half()), TypeError),
        (lambda: gpu.cnn_fc_f8_fwd(x, xs, w[:, :128].contiguous(), ws), ValueError),
        (lambda: gpu.cnn_fc_f8_fwd(x, xs, w, ws, b[:5].contiguous()), ValueError),
        (lambda: gpu.cnn_fc_f8_fwd(x, xs, w, ws, b, y_dtype=torch.float64), gpu.CnnError),
        (lambda: gpu.cnn_fc_f8_fwd(x, xs, w, ws, b, y_dtype=torch.float16, y=torch.empty((4, 130), device="cuda")), TypeError),
        (lambda: gpu.cnn_fc_f8_fwd(x, xs.cpu(), w, ws), TypeError),
        (lambda: gpu.cnn_fc_f8_fwd(x[:, ::2], xs, w, ws), ValueError),
    ]:
        with pytest.raises(error):
            call()
