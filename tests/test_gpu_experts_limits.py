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
