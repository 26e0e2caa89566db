"""Products on 8-bit floats (GPU) on every way that a call takes (``f8_ways``), by equality: sums are fp32 whatever the
result's type, so that results of 16 bits are the fp32 ones rounded, and sums that 24 bits hold are exact."""
import math

import pytest
import torch

import f8_ways
import head_ref as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
IDS = ["f32", "bf16", "f16"]
EVERY = f8_ways.ON_ROWS + f8_ways.ON_TILES


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(shape, g):
    return torch.randn(shape, generator=g, device="cuda")


def operands(n, i, o, seed):
    g, nb = gen(seed), ref.blocks_of(i)
    return (ref.random_f8((n, i), g), torch.exp(0.5 * randn((n, nb), g)) / 100, ref.random_f8((o, i), g),
            torch.exp(0.5 * randn((ref.blocks_of(o), nb), g)) / (100 * math.sqrt(i)), 0.1 * randn((o,), g))


def ones(n, i, o):
    nb = ref.blocks_of(i)
    return torch.ones((n, nb), device="cuda"), torch.ones((ref.blocks_of(o), nb), device="cuda")


def same(a, b):
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0))


@pytest.mark.parametrize("n,i,o", EVERY)
def test_16_bit_results_are_the_fp32_ones_rounded(gpu, n, i, o):
    x, xs, w, ws, b = operands(n, i, o, n + i + o)
    for relu in (False, True):
        y = gpu.cnn_fc_f8_fwd(x, xs, w, ws, b, relu)
        want, s = ref.product(x, xs, w, ws, b, relu)
        ref.assert_product(y, want, s, i, f"{n}x{i}x{o}")
        for dtype in TYPES[1:]:
            assert torch.equal(gpu.cnn_fc_f8_fwd(x, xs, w, ws, b, relu, y_dtype=dtype), y.to(dtype)), dtype


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,i,o", EVERY)
def test_a_small_product_beside_large_ones(gpu, n, i, o, dtype):
    """64 times 2^16, -2^16 and 1 next to each other: whatever the order of additions, every sum on the way is a whole
    number of 2^22 at most."""
    x, w = torch.zeros((n, i), device="cuda"), torch.zeros((o, i), device="cuda")
    for t in range(64):
        k = t * (i // 64)
        x[:, k], x[:, k + 1], x[:, k + 2] = 256.0, 256.0, 1.0
        w[:, k], w[:, k + 1], w[:, k + 2] = 256.0, -256.0, 1.0
    xs, ws = ones(n, i, o)
    y = gpu.cnn_fc_f8_fwd(x.to(ref.F8), xs, w.to(ref.F8), ws, y_dtype=dtype)
    assert bool((y == 64).all())


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,i,o", EVERY)
def test_blocks_are_added_in_32_bits(gpu, n, i, o, dtype):
    """A block's sum of 2^16 + 1, and -2^16 in the next block, in the last one, or one block of each two: a sum of fewer than
    17 bits would lose the 1."""
    nb = ref.blocks_of(i)
    xs, ws = ones(n, i, o)
    for pairs in ([(0, 1)], [(0, nb - 1)], [(k, k + 1) for k in range(0, min(nb - 1, 64), 2)]):
        x, w = torch.zeros((n, i), device="cuda"), torch.zeros((o, i), device="cuda")
        for a, b in pairs:
            last = min(128 * b + 77, i - 1)
            x[:, 128 * a + 5], x[:, 128 * a + 90], x[:, last] = 256.0, 1.0, 256.0
            w[:, 128 * a + 5], w[:, 128 * a + 90], w[:, last] = 256.0, 1.0, -256.0
        y = gpu.cnn_fc_f8_fwd(x.to(ref.F8), xs, w.to(ref.F8), ws, y_dtype=dtype)
        assert bool((y == len(pairs)).all()), pairs


@pytest.mark.parametrize("n,i,o", EVERY)
def test_small_whole_numbers_are_exact(gpu, n, i, o):
    """Values of -4 to 4 with scales of 1/2 to 2, a bias of up to 64 quarters: sums are whole numbers of quarters, 256 i + 64 of
    them at most, which are fewer than 2^24."""
    assert 256 * i + 64 < 2 ** 24
    g, nb = gen(n + i), ref.blocks_of(i)
    x = torch.randint(-4, 5, (n, i), generator=g, device="cuda").float().to(ref.F8)
    w = torch.randint(-4, 5, (o, i), generator=g, device="cuda").float().to(ref.F8)
    xs = torch.exp2(torch.randint(-1, 2, (n, nb), generator=g, device="cuda").float())
    ws = torch.exp2(torch.randint(-1, 2, (ref.blocks_of(o), nb), generator=g, device="cuda").float())
    b = torch.randint(-64, 65, (o,), generator=g, device="cuda").float() / 4
    want = ref.product(x, xs, w, ws, b, False)[0]
    for dtype in TYPES:
        for relu in (False, True):
            y = gpu.cnn_fc_f8_fwd(x, xs, w, ws, b, relu, y_dtype=dtype)
            exact = (want.clamp(min=0) if relu else want).float().to(dtype)
            assert torch.equal(y, exact), (dtype, relu)
    assert bool((want < 0).any()) and bool((want > 0).any())


@pytest.mark.parametrize("n,i,o", f8_ways.ON_TILES)
def test_nan_and_infinity_on_tiles(gpu, n, i, o):
    """In values and in scales of both operands, in the last block: they reach the sums that they are part of, and no others.
    ReLU makes NaN 0."""
    x, xs, w, ws, b = operands(n, i, o, 7)
    clean = gpu.cnn_fc_f8_fwd(x, xs, w, ws, b)
    row, out = n // 2, o // 3
    for what in ("x", "xs", "w", "ws", "xs infinite"):
        x2, xs2, w2, ws2 = x.clone(), xs.clone(), w.clone(), ws.clone()
        bad = torch.zeros((n, o), dtype=torch.bool, device="cuda")
        if what == "x":
            x2.view(torch.uint8)[row, i - 1] = 0xff
            bad[row] = True
        elif what == "w":
            w2.view(torch.uint8)[out, i - 1] = 0x7f
            bad[:, out] = True
        elif what == "ws":
            ws2[out // 128, -1] = math.nan
            bad[:, out // 128 * 128:out // 128 * 128 + 128] = True
        else:
            xs2[row, -1] = math.nan if what == "xs" else math.inf
            bad[row] = True
        y = gpu.cnn_fc_f8_fwd(x2, xs2, w2, ws2, b)
        assert torch.equal(y[~bad], clean[~bad]), what
        assert bool((~y[bad].isfinite()).all()) if what == "xs infinite" else bool(y[bad].isnan().all()), what
        for dtype in TYPES[1:]:
            assert same(gpu.cnn_fc_f8_fwd(x2, xs2, w2, ws2, b, y_dtype=dtype), y.to(dtype)), (what, dtype)
        relu = gpu.cnn_fc_f8_fwd(x2, xs2, w2, ws2, b, True)
        assert torch.equal(relu, torch.where(y > 0, y, 0.0)), what


@pytest.mark.parametrize("n,i,o", f8_ways.ON_TILES)
def test_scales_of_a_wide_range_on_tiles(gpu, n, i, o):
    """From 2^-60 to 2^60 by the block, whose product is around 1: each block's own two count."""
    x, _, w, _, _ = operands(n, i, o, 5)
    k = torch.arange(ref.blocks_of(i), device="cuda", dtype=torch.float32) % 5 * 30 - 60
    xs = (torch.exp2(k) * (1 + torch.arange(n, device="cuda").float()[:, None] / n) / (1024 * 128)).contiguous()
    ws = (torch.exp2(-k) * (1 + torch.arange(ref.blocks_of(o), device="cuda").float()[:, None])).contiguous()
    y = gpu.cnn_fc_f8_fwd(x, xs, w, ws)
    want, s = ref.product(x, xs, w, ws, None, False)
    ref.assert_product(y, want, s, i, f"{n}x{i}x{o}")
    for dtype in TYPES[1:]:
        assert torch.equal(gpu.cnn_fc_f8_fwd(x, xs, w, ws, y_dtype=dtype), y.to(dtype)), dtype


@pytest.mark.parametrize("n,i,o", [(1, 8192, 28672), (1, 4096, 32000), (16, 4096, 32000)])
def test_few_tokens_of_many_outputs(gpu, n, i, o):
    """A token's results do not depend on whether tiles or rows are quicker: 2^16, -2^16 and 1 by eights."""
    x, w = torch.zeros((n, i), dtype=torch.uint8, device="cuda"), torch.zeros((o, i), dtype=torch.uint8, device="cuda")
    for k in range(0, i, i // 64):
        x[:, k], x[:, k + 3], x[:, k + 5] = 0x78, 0x78, 0x38      # 256, 256, 1
        w[:, k], w[:, k + 3], w[:, k + 5] = 0x78, 0xf8, 0x38      # 256, -256, 1
    xs, ws = ones(n, i, o)
    for dtype in TYPES:
        y = gpu.cnn_fc_f8_fwd(x.view(ref.F8), xs, w.view(ref.F8), ws, y_dtype=dtype)
        assert bool((y == 64).all())
