"""Norm, 8-bit floats and sampling at the largest sizes that their arguments' checks allow (GPU).  Values are
exact, so that results are compared for equality."""
import pytest
import torch

pytestmark = pytest.mark.gpu

MOST = 2**31 - 1
F8 = torch.float8_e4m3fn


def behind(n, dtype, value):
    """n elements to write to, and 64 behind them that hold `value`."""
    flat = torch.full((n + 64,), value, dtype=dtype, device="cuda")
    return flat[:n], flat[n:]


def one_448():
    return torch.tensor(1.0) / torch.tensor(448.0)


def signs(n, dtype):
    """1 and -1 at random places."""
    g = torch.Generator(device="cuda")
    g.manual_seed(n % 1000)
    return torch.empty(n, dtype=torch.int8, device="cuda").random_(0, 2, generator=g).mul_(2).sub_(1).to(dtype)


@pytest.mark.parametrize("rows,cols", [(1, MOST), (1, MOST - 9), (MOST, 1), (2**24 - 1, 128), (3, MOST // 3)])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_most(gpu, rows, cols, block_rows):
    x = signs(rows * cols, torch.bfloat16)
    q, rest = behind(rows * cols, torch.uint8, 9)
    y, tail = behind(rows * cols, torch.bfloat16, 5.0)
    _, scale = gpu.cnn_f8_quantize(x.view(rows, cols), block_rows, q=q.view(F8).view(rows, cols))
    assert bool((scale == one_448()).all()) and bool((rest == 9).all())
    assert bool((q == torch.where(x > 0, 0x7e, 0xfe)).all())
    gpu.cnn_f8_dequantize(q.view(F8).view(rows, cols), scale, block_rows, y=y.view(rows, cols))
    assert torch.equal(x, y) and bool((tail == 5).all())


@pytest.mark.parametrize("rows,cols", [(1, MOST), (1, MOST - 9), (MOST, 1), (2**24 - 1, 128), (65536, 32767)])
def test_norm_most(gpu, rows, cols):
    x = signs(rows * cols, torch.float16).mul_(2)
    y, rest = behind(rows * cols, torch.float16, 9.0)
    gpu.cnn_rms_norm_fwd(x.view(rows, cols), eps=0.0, y=y.view(rows, cols))
    assert bool((rest == 9).all()) and bool((y * 2 == x).all())
    del y, rest
    q, rest = behind(rows * cols, torch.uint8, 9)
    _, scale = gpu.cnn_rms_norm_fwd(x.view(rows, cols), eps=0.0, f8=True, y=q.view(F8).view(rows, cols))
    assert bool((rest == 9).all()) and bool((scale == one_448()).all())
    assert bool((q == torch.where(x > 0, 0x7e, 0xfe)).all())


@pytest.mark.parametrize("n,i,o", [(MOST, 1, 1), (1, MOST, 1), (1, 1, MOST), (MOST - 8, 1, 1), (46340, 46340, 2), (2, 46340, 46340),
                                   (46340, 2, 46340), (2, 2**23 - 1, 256), (256, 2**23 - 1, 2), (16383, 131072, 3)])
def test_product_most(gpu, n, i, o):
    """One input and one weight of a row are not zero, at places that differ from row to row but meet at the last one."""
    x, w = torch.zeros((n, i), dtype=torch.uint8, device="cuda"), torch.zeros((o, i), dtype=torch.uint8, device="cuda")
    x[:, -1], w[:, -1] = 0x38, 0x40                     # 1 and 2
    if i > 2:
        x[:, 0], w[:, i // 2] = 0x38, 0x38              # meet zeros
    w[o // 2, -1] = 0x48                                # 4
    x[n - 1, -1] = 0x30                                # 1 / 2
    nb = (i + 127) // 128
    xs, ws = torch.ones((n, nb), device="cuda"), torch.ones(((o + 127) // 128, nb), device="cuda")
    y, rest = behind(n * o, torch.float16, 9.0)
    y = y.view(n, o)
    gpu.cnn_fc_f8_fwd(x.view(F8), xs, w.view(F8), ws, y=y)
    assert bool((rest == 9).all())
    if n > 1:
        top = y[:-1]
        assert bool((top[:, o // 2] == 4).all()) and bool((top[:, :o // 2] == 2).all()) and bool((top[:, o // 2 + 1:] == 2).all())
    assert bool((y[-1, :o // 2] == 1).all()) and float(y[-1, o // 2]) == 2 and bool((y[-1, o // 2 + 1:] == 1).all())


def test_sample_longest_row(gpu):
    """One row: all alike, and three tokens above the others."""
    x = torch.zeros((1, MOST), dtype=torch.bfloat16, device="cuda")
    for u in (0.0, 0.75, 1 - 2.0**-24):
        token, prob = gpu.cnn_sample_fwd(x, torch.tensor([u], device="cuda"))
        assert int(token) == int(u * MOST) and float(prob) == float(torch.tensor(1 / MOST))
    x[0, -1], x[0, 5], x[0, 2**30 + 3] = 200.0, 200.0, 200.0
    for kw in ({}, {"top_k": torch.tensor([3], dtype=torch.int32, device="cuda")}, {"top_p": torch.tensor([0.99], device="cuda")}):
        for u, want in ((0.2, 5), (0.5, 2**30 + 3), (0.9, MOST - 1)):
            token, prob = gpu.cnn_sample_fwd(x, torch.tensor([u], device="cuda"), **kw)
            assert int(token) == want and float(prob) == float(torch.tensor(1 / 3))


def test_sample_most_rows(gpu):
    n, v = 2**22, 511
    x = torch.zeros((n, v), dtype=torch.float16, device="cuda")
    at = torch.arange(n, device="cuda") * 7 % v
    x.scatter_(1, at[:, None], 100.0)
    u = torch.full((n,), 0.5, device="cuda")
    for k in (None, torch.full((n,), 5, dtype=torch.int32, device="cuda")):
        token, prob = gpu.cnn_sample_fwd(x, u, top_k=k)
        assert torch.equal(token.long(), at) and bool((prob == 1).all())
