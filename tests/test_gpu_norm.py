"""The root-mean-square norm with the residual's addition (GPU), in wide types
and to 8 bits, against references in 64 bits (``head_ref``)."""
import math

import pytest
import torch

import head_ref as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
IDS = ["f32", "bf16", "f16"]
SIZES = [(1, 1), (1, 7), (3, 8), (2, 127), (5, 128), (4, 129), (1, 4096), (70, 520), (77, 1013), (9, 4100), (3, 8192), (2, 16500),
         (2, 32768), (2, 32776), (1, 70001), (3000, 64)]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def inputs(rows, cols, dtype, seed):
    g = gen(seed)
    size = torch.exp(0.5 * torch.randn((cols,), generator=g, device="cuda"))
    x = (torch.randn((rows, cols), generator=g, device="cuda") * size).to(dtype)
    r = (2 * torch.randn((rows, cols), generator=g, device="cuda") * size).to(dtype)
    w = 1 + 0.3 * torch.randn((cols,), generator=g, device="cuda")
    return x, r, w


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_norm(gpu, rows, cols, dtype):
    x, r, w = inputs(rows, cols, dtype, rows + cols)
    for residual, weight in ((r, w), (None, w), (r, None), (None, None)):
        what = f"{rows}x{cols} {dtype} {residual is not None} {weight is not None}"
        s, want = ref.norm(x, residual, weight, 1e-6)
        got = gpu.cnn_rms_norm_fwd(x, weight, residual)
        y, total = got if residual is not None else (got, None)
        assert y.dtype is dtype and y.shape == x.shape
        ref.assert_norm(y, want, what)
        if residual is not None:
            assert torch.equal(total, s.to(dtype))
        got = gpu.cnn_rms_norm_fwd(x, weight, residual, f8=True)
        ref.assert_norm_f8(got[0], got[1], want, what)
        if residual is not None:
            assert torch.equal(got[2], s.to(dtype))


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("rows,cols", [(3, 300), (2, 9000), (2, 20000), (2, 40000)])
def test_norm_in_place(gpu, rows, cols, dtype):
    x, r, w = inputs(rows, cols, dtype, 3)
    y, s = gpu.cnn_rms_norm_fwd(x, w, r)
    a, b = x.clone(), r.clone()
    got = gpu.cnn_rms_norm_fwd(a, w, b, sum=b, y=a)
    assert got[0].data_ptr() == a.data_ptr() and torch.equal(a, y) and torch.equal(b, s)
    a, b = x.clone(), r.clone()
    gpu.cnn_rms_norm_fwd(a, w, b, sum=a, y=b)
    assert torch.equal(b, y) and torch.equal(a, s)
    a = x.clone()
    gpu.cnn_rms_norm_fwd(a, w, a, sum=a)            # x added to itself, in its place
    assert torch.equal(a, (2 * x.float()).to(dtype))
    a = x.clone()
    assert torch.equal(gpu.cnn_rms_norm_fwd(a, w, y=a), gpu.cnn_rms_norm_fwd(x, w))
    q, scale, _ = gpu.cnn_rms_norm_fwd(x, w, r, f8=True)
    b = r.clone()
    q2, scale2, _ = gpu.cnn_rms_norm_fwd(x, w, b, f8=True, sum=b)
    assert torch.equal(q.double(), q2.double()) and torch.equal(scale, scale2) and torch.equal(b, s)


@pytest.mark.parametrize("cols", [96, 4096, 33000])
def test_norm_of_extremes(gpu, cols):
    """Values whose squares pass fp32 at both ends, rows of zeros, infinities, NaN."""
    x = torch.randn((7, cols), generator=gen(5), device="cuda")
    x[1] *= 1e30
    x[2] *= 1e-30
    x[3] = 0
    x[4, 3] = math.inf
    x[5, cols - 1] = math.nan
    x[6] = 3e38
    y = gpu.cnn_rms_norm_fwd(x, eps=0.0)
    _, want = ref.norm(x, None, None, 0.0)
    for row in (0, 1, 2, 6):
        ref.assert_norm(y[row:row + 1], want[row:row + 1], f"row {row}")
    assert bool(y[3].isnan().all()) and bool(y[5].isnan().all())       # 0 / 0
    assert bool(y[4, 3].isnan()) and float(y[4].nan_to_num(0).abs().max()) == 0
    y = gpu.cnn_rms_norm_fwd(x, eps=1e-6)
    _, want = ref.norm(x, None, None, 1e-6)
    for row in (0, 1, 2, 3, 6):
        ref.assert_norm(y[row:row + 1], want[row:row + 1], f"eps, row {row}")
    q, scale = gpu.cnn_rms_norm_fwd(x, eps=1e-6, f8=True)
    for row in (0, 1, 2, 3, 6):
        ref.assert_norm_f8(q[row:row + 1], scale[row:row + 1], want[row:row + 1], f"f8, row {row}")
    assert bool(scale[5].isnan().all()) and float(q[5].float().abs().max()) == 0
    assert bool(scale[4, 0].isnan()) and not bool(scale[4, 1:].isnan().any())
    half = torch.full((1, cols), 60000.0, device="cuda", dtype=torch.float16)
    y, s = gpu.cnn_rms_norm_fwd(half, None, half)
    assert bool(torch.isinf(s).all()) and bool((y == 1).all())          # the norm is of the sum before it is rounded


def test_norm_is_that_of_the_unrounded_sum(gpu):
    x = torch.full((1, 256), 256.0, device="cuda", dtype=torch.bfloat16)
    r = torch.full((1, 256), 0.75, device="cuda", dtype=torch.bfloat16)
    x[0, ::2] = -256.0
    w = torch.full((256,), 256.0, device="cuda")
    y, s = gpu.cnn_rms_norm_fwd(x, w, r, eps=0.0)
    assert float(s[0, 1]) == 256.0 and float(s[0, 0]) == -255.0
    _, want = ref.norm(x, r, w, 0.0)
    ref.assert_norm(y, want, "unrounded")


def test_norm_shapes_and_refusals(gpu):
    x, r, w = inputs(12, 96, torch.bfloat16, 1)
    y = gpu.cnn_rms_norm_fwd(x, w)
    assert torch.equal(gpu.cnn_rms_norm_fwd(x.reshape(3, 4, 96), w), y.reshape(3, 4, 96))
    assert torch.equal(gpu.cnn_rms_norm_fwd(x[0], w), y[0])
    q, s = gpu.cnn_rms_norm_fwd(x.reshape(3, 4, 96), w, f8=True)
    assert q.shape == (3, 4, 96) and s.shape == (3, 4, 1)
    assert gpu.cnn_rms_norm_fwd(x[:0], w).shape == (0, 96)
    q, s, t = gpu.cnn_rms_norm_fwd(x[:0], w, r[:0], f8=True)
    assert q.shape == (0, 96) and s.shape == (0, 1) and t.shape == (0, 96)
    for call, error in [
        (lambda: gpu.cnn_rms_norm_fwd(x.double(), w), TypeError),
        (lambda: gpu.cnn_rms_norm_fwd(x.T, w), TypeError),
        (lambda: gpu.cnn_rms_norm_fwd(x, w.bfloat16()), TypeError),
        (lambda: gpu.cnn_rms_norm_fwd(x, w[:95].contiguous()), ValueError),
        (lambda: gpu.cnn_rms_norm_fwd(x, w, r.float()), TypeError),
        (lambda: gpu.cnn_rms_norm_fwd(x, w, r[:5].contiguous()), ValueError),
        (lambda: gpu.cnn_rms_norm_fwd(x, w, sum=r), ValueError),
        (lambda: gpu.cnn_rms_norm_fwd(x, w, r, sum=x, y=x), gpu.CnnError),
        (lambda: gpu.cnn_rms_norm_fwd(x, w, f8=True, y=x), TypeError),
        (lambda: gpu.cnn_rms_norm_fwd(x, w, y_scale=w), ValueError),
        (lambda: gpu.cnn_rms_norm_fwd(x, w, eps=-1.0), gpu.CnnError),
        (lambda: gpu.cnn_rms_norm_fwd(x, w, eps=math.nan), gpu.CnnError),
        (lambda: gpu.cnn_rms_norm_fwd(x[:, :0].contiguous()), ValueError),
        (lambda: gpu.cnn_rms_norm_fwd(x.cpu(), w), TypeError),
    ]:
        with pytest.raises(error):
            call()


def test_norm_writes_its_own_rows_only(gpu):
    for rows, cols in ((3, 100), (2, 33001)):
        x, r, w = inputs(rows, cols, torch.float32, 2)
        room = torch.full((rows * cols + 64,), 7.0, device="cuda")
        y = room[32:32 + rows * cols].view(rows, cols)
        gpu.cnn_rms_norm_fwd(x, w, r, y=y)
        assert bool((room[:32] == 7).all()) and bool((room[32 + rows * cols:] == 7).all())
        nb = ref.blocks_of(cols)
        qroom = torch.full((rows * cols + 64,), 7, dtype=torch.uint8, device="cuda")
        sroom = torch.full((rows * nb + 64,), 7.0, device="cuda")
        gpu.cnn_rms_norm_fwd(x, w, r, f8=True, y=qroom[33:33 + rows * cols].view(ref.F8).view(rows, cols),
                             y_scale=sroom[32:32 + rows * nb].view(rows, nb))
        assert bool((qroom[:33] == 7).all()) and bool((qroom[33 + rows * cols:] == 7).all())
        assert bool((sroom[:32] == 7).all()) and bool((sroom[32 + rows * nb:] == 7).all())


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows,cols", [(1024, 4096), (3000, 1000), (100, 33000)])
def test_norm_in_8_bits_is_that_of_unrounded_values(gpu, rows, cols, residual):
    """Among 10^6 values some are so near to the middle between two 8-bit floats that fp32's roundings would decide: codes are
    those of the definition in 64 bits, but for values within 2^-50 of a middle (of 10^6 none)."""
    g = gen(rows)
    x = torch.randn((rows, cols), generator=g, device="cuda")
    r = torch.randn((rows, cols), generator=g, device="cuda") if residual else None
    w = 1 + 0.2 * torch.randn((cols,), generator=g, device="cuda")
    q, scale = gpu.cnn_rms_norm_fwd(x, w, r, 1e-5, f8=True)[:2]
    want, want_scale = ref.quantize(ref.norm(x, r, w, 1e-5)[1])
    assert torch.equal(q.double(), want)
    assert bool(((scale.double() / want_scale.double() - 1).abs() <= 4 * 2.0 ** -24).all())


def test_norm_of_the_largest_eps(gpu):
    """eps of fp32's largest number, beside squares of 2^100 and of 2^130."""
    x, _, w = inputs(2, 200, torch.float32, 5)
    x[0] *= 2.0 ** 50
    x[1] *= 2.0 ** 65
    eps = float(torch.finfo(torch.float32).max)
    ref.assert_norm(gpu.cnn_rms_norm_fwd(x, w, eps=eps), ref.norm(x, None, w, eps)[1], "largest eps")


@pytest.mark.parametrize("dtype", TYPES[1:], ids=IDS[1:])
@pytest.mark.parametrize("rows,cols", [(4, 1000), (3, 20000), (2, 40000)])
def test_norm_is_not_that_of_the_rounded_sum(gpu, rows, cols, dtype):
    """Values at which the bounds tell the two apart: here, and for 4 x 1000 without a GPU (``test_head_abi``)."""
    x, r, w = (t.cuda() for t in ref.norm_inputs(rows, cols, dtype))
    s, want = ref.norm(x, r, w, 1e-6)
    other = ref.norm(s.to(dtype), None, w, 1e-6)[1]
    with pytest.raises(AssertionError):
        ref.assert_norm(other.to(dtype), want, "rounded")
    ref.assert_norm(gpu.cnn_rms_norm_fwd(x, w, r)[0], want, "unrounded")
    ref.assert_norm_f8(*gpu.cnn_rms_norm_fwd(x, w, r, f8=True)[:2], want, "unrounded, 8 bits")
