"""The operators on microscaled 4-bit values and on groups of rows: calls that
are refused before any launch (no GPU needed), and the references that the GPU
tests use, pinned by worked examples."""
import math

import pytest
import torch

import experts_ref as ref

cnn = pytest.importorskip("paper_1511_07376_amd.cnn", reason="libcnn.so not built")
L = cnn.lib
FAKE = 0x1000  # never dereferenced: the checks refuse first
INV, UNS, WS = cnn.CNN_ERR_INVALID, cnn.CNN_ERR_UNSUPPORTED, cnn.CNN_ERR_WORKSPACE
F32, BF16, F16, MX4 = cnn.CNN_F32, cnn.CNN_BF16, cnn.CNN_F16, cnn.CNN_MX4


@pytest.mark.parametrize("args,status", [
    # x, type, rows, cols, q, scale
    ((FAKE, MX4, 2, 32, FAKE, FAKE), INV),              # mx4 is no input
    ((FAKE, 7, 2, 32, FAKE, FAKE), INV),
    ((FAKE, F32, -1, 32, FAKE, FAKE), INV),
    ((FAKE, F32, 2, 0, FAKE, FAKE), INV),
    ((0, F32, 2, 32, FAKE, FAKE), INV),
    ((FAKE, F32, 2, 32, 0, FAKE), INV),
    ((FAKE, F32, 2, 32, FAKE, 0), INV),
    ((FAKE, F32, 70000, 70000, FAKE, FAKE), UNS),       # over 2^31-1 values
    ((FAKE + 2, F32, 2, 32, FAKE, FAKE), INV),          # fp32 at an odd half-word
    ((FAKE, F32, 2, 32, FAKE + 8, FAKE), UNS),          # q not 16-byte aligned
    ((0, BF16, 0, 32, 0, 0), cnn.CNN_OK),               # nothing to do
])
def test_mx4_conversions_refuse(args, status):
    assert L.cnn_mx4_quantize(*args, 0) == status
    x, t, rows, cols, q, s = args
    assert L.cnn_mx4_dequantize(q, s, rows, cols, x, t, 0) == status
    if status < 0:
        assert cnn.cnn_last_error().startswith("mx4_dequantize")


def _fc(**kw):
    a = dict(x=FAKE, xs=0, xt=BF16, N=4, I=64, w=FAKE, ws=FAKE, bias=0, O=8, relu=0, y=FAKE, yt=BF16, work=0, n=0, st=0)
    a.update(kw)
    return L.cnn_fc_mx4_fwd(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(x=0), INV), (dict(w=0), INV), (dict(ws=0), INV), (dict(y=0), INV),
    (dict(xs=FAKE), INV),                                # scales with wide inputs
    (dict(xt=MX4), INV),                                 # mx4 inputs without scales
    (dict(xt=5), INV), (dict(yt=F32), INV), (dict(xt=MX4, xs=FAKE, yt=MX4), INV),
    (dict(N=-1), INV), (dict(I=0), INV), (dict(O=0), INV), (dict(O=-3), INV),
    (dict(N=70000, I=70000), UNS), (dict(O=70000, I=70000), UNS), (dict(N=70000, O=70000), UNS),
    (dict(w=FAKE + 4), UNS), (dict(x=FAKE + 1), UNS), (dict(y=FAKE + 1), UNS), (dict(bias=FAKE + 2), UNS),
    (dict(xt=MX4, xs=FAKE, x=FAKE + 8, yt=F32), UNS),
    (dict(N=64, I=9216, O=4096, work=0, n=1 << 30), WS),  # a split reduction without its workspace
    (dict(N=64, I=9216, O=4096, work=FAKE, n=1024), WS), (dict(N=64, I=9216, O=4096, work=FAKE + 4, n=1 << 30), UNS),
    (dict(N=0, x=0, y=0), cnn.CNN_OK),
])
def test_fc_mx4_refuses(kw, status):
    assert _fc(**kw) == status
    if status < 0:
        assert cnn.cnn_last_error().startswith("fc_mx4")


def _grouped(**kw):
    a = dict(x=FAKE, xs=0, xt=BF16, N=4, I=64, rows=FAKE, M=6, offsets=FAKE, G=3, w=FAKE, ws=0, wt=BF16, bias=0, O=8,
             relu=0, y=FAKE, yt=BF16, work=0, n=0, st=0)
    a.update(kw)
    return L.cnn_fc_grouped_fwd(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(offsets=0), INV), (dict(x=0), INV), (dict(w=0), INV), (dict(y=0), INV), (dict(G=0), INV),
    (dict(rows=0), INV),                                 # 6 rows of y from 4 of x
    (dict(wt=F16), INV),                                 # two wide types
    (dict(xt=MX4, xs=FAKE), INV),                        # mx4 inputs, wide weights
    (dict(wt=MX4), INV), (dict(ws=FAKE), INV), (dict(yt=F16), INV),
    (dict(M=-1), INV), (dict(N=0, M=6), INV), (dict(I=0), INV),
    (dict(G=(1 << 20) + 1), UNS), (dict(G=1 << 20, O=40000, I=1, N=1, M=1), UNS), (dict(M=70000, O=70000), UNS), (dict(rows=FAKE + 2), UNS), (dict(offsets=FAKE + 1), UNS),
    (dict(M=0, N=0, x=0, y=0, rows=0), cnn.CNN_OK),
])
def test_fc_grouped_refuses(kw, status):
    assert _grouped(**kw) == status
    if status < 0:
        assert cnn.cnn_last_error().startswith("fc_grouped")


def _route(**kw):
    a = dict(logits=FAKE, t=F32, T=100, E=8, k=2, renorm=0, expert=FAKE, weight=FAKE, rows=FAKE, offsets=FAKE, slot=FAKE,
             ws=FAKE, n=1 << 20, st=0)
    a.update(kw)
    return L.cnn_route_fwd(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(t=MX4), INV), (dict(T=-1), INV), (dict(E=0), INV), (dict(k=0), INV), (dict(k=9), INV),
    (dict(E=1025), UNS), (dict(E=100, k=65), UNS), (dict(T=(1 << 26) + 1, E=1, k=1), UNS), (dict(T=1 << 25, E=1000), UNS),
    (dict(logits=0), INV), (dict(expert=0), INV), (dict(weight=0), INV), (dict(rows=0), INV), (dict(offsets=0), INV),
    (dict(slot=0), INV), (dict(logits=FAKE + 2), UNS), (dict(ws=FAKE + 2), UNS),
    (dict(ws=0), WS), (dict(n=5 * 8 * 4 - 1), WS),       # four workgroups of 32 tokens and the totals
])
def test_route_refuses(kw, status):
    assert _route(**kw) == status
    assert cnn.cnn_last_error().startswith("route")


def test_fc_workspaces():
    assert L.cnn_fc_mx4_workspace_bytes(BF16, 1, 4096, 4096) == 0
    assert 0 < L.cnn_fc_mx4_workspace_bytes(F32, 64, 9216, 4096) <= 64 << 20
    assert L.cnn_fc_mx4_workspace_bytes(7, 64, 9216, 4096) == 0 and L.cnn_fc_mx4_workspace_bytes(F32, 64, 0, 4096) == 0
    assert 0 < L.cnn_fc_grouped_workspace_bytes(BF16, 4096, 8192, 8, BF16, 4096) <= 64 << 20
    assert L.cnn_fc_grouped_workspace_bytes(BF16, 4096, 8192, 8, F16, 4096) == 0


def test_route_workspace():
    assert cnn.lib.cnn_route_workspace_bytes(64, 8, 2) == 0
    assert cnn.lib.cnn_route_workspace_bytes(65, 8, 2) == 4 * 8 * 4
    assert cnn.lib.cnn_route_workspace_bytes(65, 8, 9) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(t=MX4), INV), (dict(M=-1), INV), (dict(D=0), INV), (dict(N=-1), INV), (dict(k=0), INV), (dict(x=0), INV),
    (dict(slot=0), INV), (dict(weight=0), INV), (dict(y=0), INV), (dict(M=70000, D=70000), UNS),
    (dict(N=70000, D=70000), UNS), (dict(N=1 << 20, k=4096), UNS), (dict(x=FAKE + 2), UNS), (dict(slot=FAKE + 1), UNS),
    (dict(N=0, y=0, slot=0, weight=0), cnn.CNN_OK),
])
def test_combine_refuses(kw, status):
    a = dict(x=FAKE, t=F32, M=6, D=8, slot=FAKE, weight=FAKE, N=3, k=2, y=FAKE, st=0)
    a.update(kw)
    assert L.cnn_combine_fwd(*a.values()) == status
    if status < 0:
        assert cnn.cnn_last_error().startswith("combine")


def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 64)
    with pytest.raises(TypeError):
        cnn.cnn_mx4_quantize(x)
    with pytest.raises(TypeError):
        cnn.cnn_fc_mx4_fwd(x, x, x)
    with pytest.raises(TypeError):
        cnn.cnn_route_fwd(x, 2)
    with pytest.raises(TypeError):
        cnn.cnn_combine_fwd(x, x, x)


# ---------------------------------------------------------------- the references
def test_reference_rounding():
    """Every midpoint goes to the even code, in both signs; 4 is the block's largest, so its scale is 1."""
    x = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 0.2500001, -0.25, -0.75, 0.7499, 0.0, -3.4999] + [0.0] * 19
    q, s = ref.quantize(torch.tensor([x]))
    assert s.tolist() == [[127]]
    assert ref.values(q, s, 13)[0].tolist() == [4, 0, 1, 1, 2, 2, 4, 0.5, -0.0, -1, 0.5, 0, -3]
    q, s = ref.quantize(torch.tensor([[5.0, 7.99, 6.5] + [0.0] * 29]))
    assert s.tolist() == [[127]] and ref.values(q, s, 3)[0].tolist() == [4, 6, 6]


def test_reference_scales():
    x = torch.zeros(5, 32)
    x[1, 3], x[2, 0], x[3, 31], x[4, 1] = 2.0 ** -149, 3.4e38, math.inf, 1.0
    q, s = ref.quantize(x)
    assert s.flatten().tolist() == [0, 0, 252, 255, 125]
    assert ref.values(q, s, 32)[1].abs().max() == 0


def test_reference_route():
    inf, nan = math.inf, math.nan
    logits = torch.tensor([[1.0, 3.0, 3.0, 0.0], [-inf, -inf, 2.0, -inf], [-inf, -inf, -inf, nan], [0.0, -0.0, nan, -1.0]])
    expert, weight, rows, offsets, slot = ref.route(logits, 2, True)
    assert expert.tolist() == [[1, 2], [2, -1], [-1, -1], [0, 1]]
    assert weight.tolist() == [[0.5, 0.5], [1.0, 0.0], [0.0, 0.0], [0.5, 0.5]]
    assert offsets.tolist() == [0, 1, 3, 5, 5]
    assert rows.tolist() == [3, 0, 3, 0, 1, -1, -1, -1]
    assert slot.tolist() == [[1, 3], [4, -1], [-1, -1], [0, 2]]
