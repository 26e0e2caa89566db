"""Wide inputs of products on 4-bit weights keep all their bits: pairs of values that cancel but for their last bits.

A row of x is zero but for v at one column and 1 at another, which meet weights of 1 and -1: the result is v - 1.  The
bfloat16 parts of v, their products and every partial sum of them (v's parts, -1, in any order) are multiples of 2^-23
below 2, or 2^-23 itself: numbers of 24 bits, exact in fp32 whether sums are rounded or cut.  So results are compared
for equality."""
import pytest
import torch

# what a value needs of its bits: the last one of fp32, some in the middle, both, the last one of fp16
FP32 = [1 + 2.0 ** -23, 1 + 2.0 ** -12, 1 + 2.0 ** -8 + 2.0 ** -16, 1 + 2.0 ** -15, 1 + 2.0 ** -16, 2 - 2.0 ** -23]
FP16 = [1 + 2.0 ** -10, 1 + 2.0 ** -8, 2 - 2.0 ** -10]


def operands(values, n, i, o, device):
    """x [n][i] (float64), w (bytes) and scales of [o][i], and x w^T: row r holds values[r % len], its columns move
    with the row."""
    blocks = -(-i // 32)
    a = (7 * torch.arange(n, device=device)) % (i // 2) * 2     # even columns: +1
    b = (11 * torch.arange(n, device=device) + 3) % (i // 2) * 2 + 1
    v = torch.tensor(values, dtype=torch.float64, device=device)[torch.arange(n, device=device) % len(values)]
    x = torch.zeros((n, i), dtype=torch.float64, device=device)
    at = torch.arange(n, device=device)
    x[at, a], x[at, b] = v, 1.0
    w = torch.zeros((o, blocks * 16), dtype=torch.uint8, device=device)
    w[:, :i // 2] = 0x2 | 0xA << 4                              # +1, -1, +1, ...
    scale = torch.full((o, blocks), 127, dtype=torch.uint8, device=device)
    return x, w, scale, (v - 1).unsqueeze(1).expand(n, o)


def assert_kept(y, want):
    assert torch.equal(y.double(), want), f"off by {float((y.double() - want).abs().max()):.3g}"


def product_of_parts(x, parts):
    """The operation as the kernels do it, on `parts` bfloat16 parts of x (fp32), least first, summed in fp32."""
    rest, cut = x.float(), []
    for _ in range(parts):
        lead = (rest.view(torch.int32) & -65536).view(torch.float32)
        cut.append(lead)
        rest = rest - lead
    sign = 1.0 - 2.0 * (torch.arange(x.shape[1]) % 2)
    y = torch.zeros(x.shape[0])
    for part in reversed(cut):
        for c in range(x.shape[1]):
            y = y + part[:, c] * sign[c]
    return y.unsqueeze(1)


@pytest.mark.parametrize("values,needed", [(FP32, 3), (FP16, 2)], ids=["f32", "f16"])
def test_fewer_parts_are_seen(values, needed):
    """Inputs of which a part is left out do not pass, for each number of parts (no GPU needed)."""
    x, _, _, want = operands(values, 12, 64, 1, "cpu")
    assert_kept(product_of_parts(x, needed), want)
    for parts in range(needed):
        with pytest.raises(AssertionError):
            assert_kept(product_of_parts(x, parts), want)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 3, 9, 20, 40, 200])
@pytest.mark.parametrize("i,o", [(64, 20), (610, 150), (2048, 1500)])
@pytest.mark.parametrize("dtype,values", [(torch.float32, FP32), (torch.float16, FP16)], ids=["f32", "f16"])
def test_fc_mx4_keeps_the_last_bits(gpu, dtype, values, i, o, n):
    x, w, scale, want = operands(values, n, i, o, "cuda")
    assert_kept(gpu.cnn_fc_mx4_fwd(x.to(dtype), w, scale), want)


@pytest.mark.gpu
@pytest.mark.parametrize("each", [2, 12, 40, 300])
@pytest.mark.parametrize("dtype,values", [(torch.float32, FP32), (torch.float16, FP16)], ids=["f32", "f16"])
def test_fc_grouped_keeps_the_last_bits(gpu, dtype, values, each):
    i, o, groups = 610, 150, 3
    x, w, scale, want = operands(values, each * groups, i, o, "cuda")
    offsets = torch.arange(groups + 1, dtype=torch.int32, device="cuda") * each
    y = gpu.cnn_fc_grouped_fwd(x.to(dtype), w.repeat(groups, 1, 1), offsets, w_scale=scale.repeat(groups, 1, 1))
    assert_kept(y, want)
