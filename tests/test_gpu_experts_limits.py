"""The operators on 4-bit values and on groups of rows at the largest sizes that their arguments' checks allow (GPU).
Values are exact, so that results are compared for equality."""
import pytest
import torch

pytestmark = pytest.mark.gpu

MOST = 2**31 - 1


def behind(n, dtype, value):
    """n elements to write to, and 64 behind them that hold `value`."""
    flat = torch.full((n + 64,), value, dtype=dtype, device="cuda")
    return flat[:n], flat[n:]


@pytest.mark.parametrize("o", [MOST, MOST - 1, MOST - 15])
def test_fc_grouped_most_outputs(gpu, o):
    x = torch.full((1, 1), 2.0, dtype=torch.bfloat16, device="cuda")
    w = torch.ones((1, o, 1), dtype=torch.bfloat16, device="cuda")
    w[0, -40:, 0] = torch.arange(1, 41, device="cuda")
    y, rest = behind(o, torch.bfloat16, -1.0)
    y = y.view(1, o)
    gpu.cnn_fc_grouped_fwd(x, w, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), y=y)
    assert torch.equal(y[0, -40:], 2 * w[0, -40:, 0])
    assert bool((y[0, :-40] == 2).all()) and bool((rest == -1).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("cols", [MOST, MOST - 1, MOST - 7, MOST - 30])
def test_mx4_longest_row(gpu, dtype, cols):
    """One row, to mx4 and back, as its two halves are."""
    g = torch.Generator(device="cuda")
    g.manual_seed(cols % 100)
    x = torch.empty((1, cols), dtype=dtype, device="cuda").normal_(generator=g)
    q, scale = gpu.cnn_mx4_quantize(x)
    y, rest = behind(cols, dtype, -1.0)
    gpu.cnn_mx4_dequantize(q, scale, cols, y=y.view(1, cols))
    assert bool((rest == -1).all())
    half = 2**30
    for lo, hi in ((0, half), (half, cols)):
        part = x[0, lo:hi].unsqueeze(0)
        pq, ps = gpu.cnn_mx4_quantize(part)
        assert torch.equal(q[:, lo // 2:lo // 2 + pq.shape[1]], pq)
        assert torch.equal(scale[:, lo // 32:lo // 32 + ps.shape[1]], ps)
        assert torch.equal(y[lo:hi].unsqueeze(0), gpu.cnn_mx4_dequantize(pq, ps, hi - lo, dtype=dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [MOST, MOST - 2, MOST - 3, MOST - 7])
def test_combine_longest_row(gpu, dtype, d):
    g = torch.Generator(device="cuda")
    g.manual_seed(d % 100)
    x = torch.empty((1, d), dtype=dtype, device="cuda").normal_(generator=g)
    y, rest = behind(d, dtype, -1.0)
    gpu.cnn_combine_fwd(x, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.full((1, 1), 0.5, device="cuda"),
                        y=y.view(1, d))
    assert bool((rest == -1).all())
    assert torch.equal(y, x[0].mul_(0.5))


@pytest.mark.parametrize("kind", ["bf16", "mx4 on 4 bits", "bf16 on 4 bits"])
def test_fc_grouped_longest_reduction(gpu, kind):
    """One row of x, 40 times, through one of weights: tiles.  Whole blocks of the longest row are 2^31 values."""
    m, cols = 40, MOST
    offsets = torch.tensor([0, m], dtype=torch.int32, device="cuda")
    rows = torch.zeros(m, dtype=torch.int32, device="cuda")
    blocks = -(-cols // 32)
    y = torch.full((m, 1), -1.0, dtype=torch.bfloat16, device="cuda")
    # x: 1 at a few places, -1 at the last value; 4-bit codes of 1 and -1 are 2 and 10
    ones = [0, 1, 2**30 - 1, 2**30, 2**30 + 77, MOST - 40, MOST - 32, MOST - 31, MOST - 2]
    if kind == "mx4 on 4 bits":
        x = torch.zeros((1, blocks * 16), dtype=torch.uint8, device="cuda")
        for c in ones:
            x[0, c // 2] += 2 << (4 * (c % 2))
        x[0, (cols - 1) // 2] += 10 << (4 * ((cols - 1) % 2))
        xs = torch.full((1, blocks), 127, dtype=torch.uint8, device="cuda")
        x_type = gpu.CNN_MX4
    else:
        x = torch.zeros((1, cols), dtype=torch.bfloat16, device="cuda")
        x[0, ones] = 1
        x[0, -1] = -1
        xs, x_type = None, gpu.CNN_BF16
    if kind == "bf16":
        w = torch.ones((1, 1, cols), dtype=torch.bfloat16, device="cuda")
        ws, w_type = None, gpu.CNN_BF16
        w[0, 0, -1] = 4
    else:
        w = torch.full((1, 1, blocks * 16), 0x22, dtype=torch.uint8, device="cuda")
        ws, w_type = torch.full((1, 1, blocks), 127, dtype=torch.uint8, device="cuda"), gpu.CNN_MX4
        w[0, 0, -1] = 0x06                            # 4, and nothing behind the last column
    need = gpu.lib.cnn_fc_grouped_workspace_bytes(x_type, cols, m, 1, w_type, 1)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    pointer = lambda t: None if t is None else t.data_ptr()
    # the binding knows the columns of 4-bit rows as whole blocks only
    status = gpu.lib.cnn_fc_grouped_fwd(pointer(x), pointer(xs), x_type, 1, cols, pointer(rows), m, pointer(offsets), 1,
                                        pointer(w), pointer(ws), w_type, None, 1, 0, pointer(y), gpu.CNN_BF16,
                                        pointer(work), need, torch.cuda.current_stream().cuda_stream)
    assert status == gpu.CNN_OK
    assert y.flatten().tolist() == [len(ones) - 4.0] * m


def test_sizes_no_int_holds_are_refused_without_elements(gpu):
    """Tensors of no elements can have any width: it is not cut to the width that an int takes of it."""
    slot, weight = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.ones((1, 1), device="cuda")
    with pytest.raises(gpu.CnnError):
        gpu.cnn_combine_fwd(torch.empty((0, 2**32 + 8), dtype=torch.bfloat16, device="cuda"), slot, weight)
    with pytest.raises(gpu.CnnError):
        gpu.cnn_route_fwd(torch.empty((0, 2**32 + 8), device="cuda"), 2)
    with pytest.raises(gpu.CnnError):
        gpu.cnn_route_fwd(torch.empty((0, 8), device="cuda"), 2**32 + 2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_fc_grouped_most_rows(gpu, dtype):
    """2^31 - 1 rows of results, gathered from a thousand, in groups that end anywhere."""
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = torch.randint(-8, 9, (1000, 1), generator=g, device="cuda").to(dtype)
    w = torch.tensor([1.0, 2.0, 4.0], device="cuda").to(dtype).view(3, 1, 1)
    rows = torch.randint(0, 1000, (MOST,), generator=g, device="cuda", dtype=torch.int32)
    bounds = [0, 5, 2**30 + 1, MOST - 3]
    y, rest = behind(MOST, dtype, -1.0)
    gpu.cnn_fc_grouped_fwd(x, w, torch.tensor(bounds, dtype=torch.int32, device="cuda"), rows=rows, y=y.view(MOST, 1))
    assert bool((rest == -1).all()) and bool((y[MOST - 3:] == -1).all())
    for k, (lo, hi) in enumerate(zip(bounds, bounds[1:])):
        for at in range(lo, hi, 2**28):
            end = min(at + 2**28, hi)
            assert torch.equal(y[at:end], x[:, 0][rows[at:end].long()] * w[k, 0, 0]), (k, at)
