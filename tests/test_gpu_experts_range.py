"""Products on groups of rows and on 4-bit weights at the ends of their range (GPU): the smallest and the largest
scales, subnormal operands, NaN blocks, against references in 64 bits (``experts_ref``)."""
import math

import pytest
import torch

import experts_ref as ref

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(shape, g):
    return torch.randn(shape, generator=g, device="cuda")


def weights(o, i, scale, g):
    """4-bit weights of random codes, zeros behind the last column, every block of one scale."""
    w, ws = ref.random_mx4((o,), i, g)
    return w, torch.full_like(ws, scale)


def assert_bound(got, want, s, n, lost, what):
    """As experts_ref.assert_product's first bound, with `lost`: what the operands' own range may cost."""
    half = torch.finfo(got.dtype).eps / 2
    tiny = torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps
    bound = half * want.abs() + (n + 2) * 2.0 ** -23 * s * (1 + half) + lost + tiny
    err = (got.double() - want).abs()
    assert bool(torch.isfinite(err).all()), f"{what}: not finite"
    worst = float((err / bound).max())
    assert worst <= 1, f"{what}: error {worst:.3g} of its bound"


# rows: one, some and many, for the stream of weights and for each tile
ROWS = [1, 12, 20, 70, 300]


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("scale", [0, 1, 2, 3, 120, 250, 251, 252])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_fc_mx4_ends_of_the_scales(gpu, dtype, scale, n):
    """Weights down to subnormal numbers (0.5 * 2^-127) and up to 6 * 2^125; inputs of a size that brings the results
    back to about 1, but not below 2^-100, so that fp32 inputs keep all their bits."""
    g = gen(scale + n)
    i, o = 300, 150
    w, ws = weights(o, i, scale, g)
    # 2^120 at most: a normal number may be above 2, and 2 * 2^127 is infinite
    x = (randn((n, i), g).clamp(min=0.01) * 2.0 ** min(max(127 - scale, -100), 120)).to(dtype)
    want, s = ref.product(x, ref.values(w, ws, i), None, False)
    assert_bound(gpu.cnn_fc_mx4_fwd(x, w, ws), want, s, i, 0.0, f"{dtype} scale {scale} n {n}")


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("e", [-105, -110, -120, -126, -130, -140])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_fc_mx4_small_inputs(gpu, dtype, e, n):
    """Inputs around 2^e, some of them subnormal, against weights around 2^110.  bf16 inputs are exact; fp32 ones
    below 2^-107 are taken to 2^-133."""
    g = gen(n - e)
    i, o = 300, 150
    w, ws = weights(o, i, 237, g)
    x = (randn((n, i), g).double() * 2.0 ** e).to(dtype)
    wv = ref.values(w, ws, i)
    want, s = ref.product(x, wv, None, False)
    lost = 2.0 ** -133 * wv.abs().sum(1) if dtype == F32 else 0.0
    assert_bound(gpu.cnn_fc_mx4_fwd(x, w, ws), want, s, i, lost, f"{dtype} 2^{e} n {n}")


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("e", [-16, -20, -24])
def test_fc_mx4_small_fp16_inputs(gpu, e, n):
    g = gen(n - e)
    i, o = 300, 150
    w, ws = weights(o, i, 127 + 10, g)
    x = (randn((n, i), g) * 2.0 ** e).to(F16)
    want, s = ref.product(x, ref.values(w, ws, i), None, False)
    assert_bound(gpu.cnn_fc_mx4_fwd(x, w, ws), want, s, i, 0.0, f"2^{e} n {n}")


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("scales", [(0, 254), (254, 0), (1, 250), (250, 1), (60, 190), (100, 0), (0, 130), (127, 245), (245, 127)])
def test_fc_mx4_of_mx4_inputs_ends_of_the_scales(gpu, scales, n):
    """Scales whose product is in range, at every size."""
    g = gen(sum(scales) + n)
    i, o = 300, 150
    w, ws = weights(o, i, scales[1], g)
    x, xs = weights(n, i, scales[0], g)
    want, s = ref.product(ref.values(x, xs, i), ref.values(w, ws, i), None, False)
    # where all of a sum is below 2^-126, every one of its additions is rounded to, or cut at, a multiple of 2^-149
    lost = i * 2.0 ** -149
    assert_bound(gpu.cnn_fc_mx4_fwd(x, w, ws, x_scale=xs), want, s, i, lost, f"{scales} n {n}")


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("i", [32, 300, 2100])
def test_fc_mx4_of_mx4_inputs_nan_blocks(gpu, i, n):
    """A NaN block (of zeros: the scale alone makes it NaN) reaches its own row or column, and no other."""
    g = gen(i + n)
    o = 150
    w, ws = ref.random_mx4((o,), i, g)
    x, xs = ref.random_mx4((n,), i, g)
    good = gpu.cnn_fc_mx4_fwd(x, w, ws, x_scale=xs)
    assert bool(torch.isfinite(good).all())
    blocks = ws.shape[1]
    for block in sorted({0, blocks // 2, blocks - 1}):
        w2, ws2, x2, xs2 = w.clone(), ws.clone(), x.clone(), xs.clone()
        w2[33, block * 16:block * 16 + 16] = 0
        ws2[33, block] = 255
        x2[n // 2, block * 16:block * 16 + 16] = 0
        xs2[n // 2, block] = 255
        y = gpu.cnn_fc_mx4_fwd(x, w2, ws2, x_scale=xs)
        keep = torch.arange(o, device="cuda") != 33
        assert bool(torch.isnan(y[:, 33]).all()) and torch.equal(y[:, keep], good[:, keep])
        y = gpu.cnn_fc_mx4_fwd(x2, w, ws, x_scale=xs2)
        keep = torch.arange(n, device="cuda") != n // 2
        assert bool(torch.isnan(y[n // 2]).all()) and torch.equal(y[keep], good[keep])


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("e,dtype", [(-20, F16), (-24, F16), (-126, BF16), (-130, BF16), (-126, F32), (-140, F32)])
def test_fc_grouped_subnormal_operands(gpu, dtype, e, n):
    """Wide inputs around 2^e, some or all of them subnormal, against weights that bring the results into range; and
    the other way round."""
    g = gen(n - e)
    i, o = 300, 150
    small = lambda rows: (randn((rows, i), g).double() * 2.0 ** e).to(dtype)
    large = lambda rows: (randn((rows, i), g).double() * 2.0 ** min(-e - 3, 10 if dtype == F16 else 120)).to(dtype)
    offsets = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    for x, w in ((small(n), large(o)), (large(n), small(o))):
        want, s = ref.product(x, w, None, False)
        y = gpu.cnn_fc_grouped_fwd(x, w.reshape(1, o, i), offsets)
        assert_bound(y, want, s, i, 0.0, f"{dtype} 2^{e} n {n}")


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("scale", [253, 254])
def test_fc_mx4_weights_above_the_range(gpu, dtype, scale, n):
    """Beside wide inputs a weight of 2^128 or more is not finite, and no output that has one is; all others are what
    they are without it.  What is below 2^128 is held."""
    g = gen(n)
    i, o = 300, 70
    w, ws = ref.random_mx4((o,), i, g)
    x = randn((n, i), g).to(dtype)
    good = gpu.cnn_fc_mx4_fwd(x, w, ws)
    w2, ws2 = w.clone(), ws.clone()
    w2[33, 3 * 16:4 * 16] = 0
    w2[33, 3 * 16] = 6                                # one code of 4, the rest of the block zero
    ws2[33, 3] = scale
    y = gpu.cnn_fc_mx4_fwd(x, w2, ws2)
    keep = torch.arange(o, device="cuda") != 33
    assert torch.equal(y[:, keep], good[:, keep])
    assert not bool(torch.isfinite(y[:, 33]).any())
    w2[33, 3 * 16] = 3 if scale == 254 else 5        # 1.5 * 2^127 and 3 * 2^126, the largest
    x2 = torch.zeros_like(x)
    x2[:, 96] = 2.0 ** -14
    y = gpu.cnn_fc_mx4_fwd(x2, w2, ws2)
    want = 1.5 * 2.0 ** 113
    assert bool((y[:, 33].float() == (math.inf if dtype == F16 else want)).all())
