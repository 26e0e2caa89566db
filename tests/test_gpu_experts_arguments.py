"""Arguments of the operators on 4-bit values and on groups of rows that say two things (GPU)."""
import pytest
import torch

import experts_ref as ref

pytestmark = pytest.mark.gpu


def operands():
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn((3, 64), generator=g, device="cuda").bfloat16()
    w, ws = ref.random_mx4((2, 8), 64, g)
    return x, w, ws, torch.tensor([0, 1, 3], dtype=torch.int32, device="cuda")


def test_output_type_of_wide_inputs(gpu):
    """The output of wide inputs is of their type: another one is refused, the same one taken."""
    x, w, ws, offsets = operands()
    for dtype in (torch.float32, torch.float16, torch.int32):
        with pytest.raises(TypeError):
            gpu.cnn_fc_mx4_fwd(x, w[0], ws[0], y_dtype=dtype)
        with pytest.raises(TypeError):
            gpu.cnn_fc_grouped_fwd(x, w, offsets, w_scale=ws, y_dtype=dtype)
    assert torch.equal(gpu.cnn_fc_mx4_fwd(x, w[0], ws[0], y_dtype=torch.bfloat16), gpu.cnn_fc_mx4_fwd(x, w[0], ws[0]))
    assert torch.equal(gpu.cnn_fc_grouped_fwd(x, w, offsets, w_scale=ws, y_dtype=torch.bfloat16),
                       gpu.cnn_fc_grouped_fwd(x, w, offsets, w_scale=ws))


def test_output_type_of_dequantised_values(gpu):
    """A type and an output of another type: refused; without a type the output's counts."""
    _, w, ws, _ = operands()
    out = torch.empty((2, 8, 64), dtype=torch.float16, device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        with pytest.raises(TypeError):
            gpu.cnn_mx4_dequantize(w, ws, 64, dtype=dtype, y=out)
    assert gpu.cnn_mx4_dequantize(w, ws, 64, dtype=torch.float16, y=out) is out
    assert torch.equal(gpu.cnn_mx4_dequantize(w, ws, 64, y=torch.zeros_like(out)), out)
    assert gpu.cnn_mx4_dequantize(w, ws).dtype == torch.float32
