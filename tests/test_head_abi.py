"""The norm, products on 8-bit floats and sampling: calls that are refused before
any launch (no GPU needed), and the references that the GPU tests use, pinned by
worked examples."""
import math

import pytest
import torch

import head_ref as ref

cnn = pytest.importorskip("paper_1511_07376_amd.cnn", reason="libcnn.so not built")
L = cnn.lib
FAKE = 0x1000  # never dereferenced: the checks refuse first
INV, UNS, WS, OK = cnn.CNN_ERR_INVALID, cnn.CNN_ERR_UNSUPPORTED, cnn.CNN_ERR_WORKSPACE, cnn.CNN_OK
F32, BF16, F16, MX4, F8 = cnn.CNN_F32, cnn.CNN_BF16, cnn.CNN_F16, cnn.CNN_MX4, cnn.CNN_F8


@pytest.mark.parametrize("args,status", [
    # x, type, rows, cols, block_rows, q, scale
    ((FAKE, F8, 2, 32, 1, FAKE, FAKE), INV),
    ((FAKE, 9, 2, 32, 1, FAKE, FAKE), INV),
    ((FAKE, F32, -1, 32, 1, FAKE, FAKE), INV),
    ((FAKE, F32, 2, 0, 1, FAKE, FAKE), INV),
    ((FAKE, F32, 2, 32, 64, FAKE, FAKE), INV),
    ((FAKE, F32, 2, 32, 0, FAKE, FAKE), INV),
    ((0, F32, 2, 32, 1, FAKE, FAKE), INV),
    ((FAKE, F32, 2, 32, 1, 0, FAKE), INV),
    ((FAKE, F32, 2, 32, 128, FAKE, 0), INV),
    ((FAKE, F32, 70000, 70000, 1, FAKE, FAKE), UNS),
    ((FAKE + 2, F32, 2, 32, 1, FAKE, FAKE), UNS),
    ((FAKE, F32, 2, 32, 1, FAKE, FAKE + 2), UNS),
    ((0, BF16, 0, 32, 128, 0, 0), OK),
])
def test_conversions_refuse(args, status):
    assert L.cnn_f8_quantize(*args, 0) == status
    x, t, rows, cols, br, q, s = args
    assert L.cnn_f8_dequantize(q, s, rows, cols, br, x, t, 0) == status
    if status < 0:
        assert cnn.cnn_last_error().startswith("f8_dequantize")


def _norm(**kw):
    a = dict(x=FAKE, res=0, t=BF16, rows=3, cols=64, w=0, eps=1e-6, sum=0, y=FAKE + 0x100, yt=BF16, ys=0, st=0)
    a.update(kw)
    return L.cnn_rms_norm_fwd(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(x=0), INV), (dict(y=0), INV), (dict(t=F8, yt=F8, ys=FAKE), INV), (dict(t=7), INV), (dict(yt=F32), INV),
    (dict(yt=MX4), INV), (dict(yt=F8), INV), (dict(ys=FAKE), INV), (dict(rows=-1), INV), (dict(cols=0), INV),
    (dict(eps=-1e-6), INV), (dict(eps=math.nan), INV), (dict(eps=math.inf), INV),
    (dict(sum=FAKE + 0x100), INV),                        # y and sum in one place
    (dict(yt=F8, ys=FAKE, y=FAKE), INV), (dict(res=FAKE + 2, yt=F8, ys=FAKE, y=FAKE + 2), INV),
    (dict(rows=70000, cols=70000), UNS), (dict(x=FAKE + 1), UNS), (dict(res=FAKE + 1), UNS), (dict(sum=FAKE + 1), UNS),
    (dict(y=FAKE + 1), UNS), (dict(w=FAKE + 2), UNS), (dict(yt=F8, ys=FAKE + 2), UNS),
    (dict(rows=0, x=0, y=0), OK), (dict(rows=0, x=0, y=0, yt=F8), OK),
])
def test_norm_refuses(kw, status):
    assert _norm(**kw) == status
    if status < 0:
        assert cnn.cnn_last_error().startswith("rms_norm")


@pytest.mark.parametrize("eps", [0.0, 2.0 ** -149, 3.4e38, 3.4028234663852886e38])
def test_norm_takes_every_finite_eps(eps):
    """Up to fp32's largest number."""
    assert _norm(eps=eps, rows=0, x=0, y=0) == OK


def _fc(**kw):
    a = dict(x=FAKE, xs=FAKE, N=4, I=64, w=FAKE, ws=FAKE, bias=0, O=8, relu=0, y=FAKE, yt=BF16, work=0, n=0, st=0)
    a.update(kw)
    return L.cnn_fc_f8_fwd(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(x=0), INV), (dict(xs=0), INV), (dict(w=0), INV), (dict(ws=0), INV), (dict(y=0), INV), (dict(yt=F8), INV),
    (dict(yt=5), INV), (dict(N=-1), INV), (dict(I=0), INV), (dict(O=0), INV), (dict(N=70000, I=70000), UNS),
    (dict(O=70000, I=70000), UNS), (dict(N=70000, O=70000), UNS), (dict(xs=FAKE + 2), UNS), (dict(ws=FAKE + 1), UNS),
    (dict(bias=FAKE + 2), UNS), (dict(y=FAKE + 1), UNS), (dict(yt=F32, y=FAKE + 2), UNS),
    (dict(N=0, x=0, xs=0, y=0), OK),
])
def test_fc_refuses(kw, status):
    assert _fc(**kw) == status
    if status < 0:
        assert cnn.cnn_last_error().startswith("fc_f8")


def _sample(**kw):
    a = dict(x=FAKE, t=F32, N=4, V=64, u=FAKE, temp=0, k=0, p=0, m=0, token=FAKE, prob=0, work=FAKE, n=1 << 30, st=0)
    a.update(kw)
    return L.cnn_sample_fwd(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(x=0), INV), (dict(u=0), INV), (dict(token=0), INV), (dict(t=F8), INV), (dict(t=-1), INV), (dict(N=-1), INV),
    (dict(V=0), INV), (dict(N=70000, V=70000), UNS), (dict(x=FAKE + 2), UNS), (dict(u=FAKE + 2), UNS),
    (dict(temp=FAKE + 1), UNS), (dict(k=FAKE + 2), UNS), (dict(p=FAKE + 2), UNS), (dict(m=FAKE + 2), UNS),
    (dict(token=FAKE + 2), UNS), (dict(prob=FAKE + 2), UNS), (dict(work=FAKE + 4), UNS), (dict(N=0, x=0, u=0, token=0), OK),
])
def test_sample_refuses(kw, status):
    assert _sample(**kw) == status
    if status < 0:
        assert cnn.cnn_last_error().startswith("sample")


def test_workspaces_of_what_is_refused():
    assert L.cnn_fc_f8_workspace_bytes(0, 64, 64) == 0
    assert L.cnn_fc_f8_workspace_bytes(-1, 64, 64) == 0
    assert L.cnn_fc_f8_workspace_bytes(70000, 70000, 64) == 0
    assert L.cnn_sample_workspace_bytes(F8, 4, 64) == 0
    assert L.cnn_sample_workspace_bytes(F32, 0, 64) == 0
    assert L.cnn_sample_workspace_bytes(F32, 70000, 70000) == 0
    for n, i, o in [(1, 128, 128), (64, 9216, 4096), (4096, 8192, 8192), (33, 1000, 99)]:
        assert 0 <= L.cnn_fc_f8_workspace_bytes(n, i, o) <= 64 << 20


# ---------------------------------------------------------------- the references
def test_reference_f8_is_torchs_type():
    v = torch.linspace(-460, 460, 200001, dtype=torch.float64)
    v = torch.cat([v, v / 2 ** 12, torch.tensor([2.0 ** -10, 3 * 2.0 ** -10, 17.0, 19.0, 0.0, -2.0 ** -11])])
    assert torch.equal(ref.nearest_f8(v), v.clamp(-448, 448).float().to(ref.F8).double())


def test_reference_quantize():
    x = torch.zeros((2, 130))
    x[0, 0], x[0, 5], x[0, 129] = 896.0, -3.0, 2.0 ** -120
    x[1, 7], x[1, 128] = math.inf, -7.0
    q, s = ref.quantize(x)
    assert s[0, 0] == 2.0 and q[0, 0] == 448 and q[0, 5] == -1.5
    assert s[0, 1] == torch.tensor(2.0 ** -100) / 448 and q[0, 129] == nearest(2.0 ** -120 * 448 * 2.0 ** 100)
    assert math.isnan(s[1, 0]) and float(q[1, :128].abs().max()) == 0 and q[1, 128] == -448
    q, s = ref.quantize(x[:1], 128)
    assert s.shape == (1, 2) and s[0, 0] == 2.0


def nearest(v):
    return float(ref.nearest_f8(torch.tensor(v, dtype=torch.float64)))


def test_reference_norm():
    x = torch.tensor([[3.0, 4.0]])
    s, y = ref.norm(x, torch.tensor([[0.0, 0.0]]), torch.tensor([1.0, 2.0]), 0.0)
    want = torch.tensor([[3.0, 8.0]], dtype=torch.float64) / math.sqrt(12.5)
    assert torch.allclose(y, want, rtol=1e-15, atol=0) and torch.equal(s, x)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
def test_norm_bounds_see_a_sum_that_is_rounded_first(dtype):
    """The norm is of x + residual as it is before it is rounded to x's type: results of the rounded sum are outside the bounds,
    in the wide type and in 8 bits, results of the unrounded one are within."""
    x, r, w = ref.norm_inputs(4, 1000, dtype)
    s, want = ref.norm(x, r, w, 1e-6)
    other = ref.norm(s.to(dtype), None, w, 1e-6)[1]
    ref.assert_norm(want.to(dtype), want, "unrounded")
    ref.assert_norm_f8(*ref.quantize(want), want, "unrounded")
    with pytest.raises(AssertionError):
        ref.assert_norm(other.to(dtype), want, "rounded")
    with pytest.raises(AssertionError):
        ref.assert_norm_f8(*ref.quantize(other), want, "rounded")


def test_reference_product():
    g = torch.Generator().manual_seed(3)
    x, w = ref.random_f8((3, 150), g), ref.random_f8((130, 150), g)
    xs, ws = torch.rand((3, 2), generator=g), torch.rand((2, 2), generator=g)
    y, s = ref.product(x, xs, w, ws, None, False)
    n, o = 2, 129
    want = sum(float(x[n, i]) * float(xs[n, i // 128]) * float(w[o, i]) * float(ws[o // 128, i // 128]) for i in range(150))
    assert abs(float(y[n, o]) - want) < 1e-9 * float(s[n, o])


def test_reference_sample():
    x = torch.log(torch.tensor([[0.1, 0.4, 0.2, 0.3]]).double())
    one = torch.ones(1)

    def token(u, **kw):
        t, p, _ = ref.sample(x, torch.tensor([u]), **{k: torch.tensor([v]) for k, v in kw.items()})
        return int(t), float(p)
    assert [token(u)[0] for u in (0.0, 0.05, 0.15, 0.49, 0.51, 0.69, 0.71, 0.999)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert token(0.5)[1] == pytest.approx(0.4) or token(0.5)[1] == pytest.approx(0.2)
    assert token(0.0, top_k=2) == (1, pytest.approx(4 / 7)) and token(0.9, top_k=2) == (3, pytest.approx(3 / 7))
    assert token(0.99, top_p=0.41) == (3, pytest.approx(3 / 7))      # 0.4 stand before the second: less than 0.41
    assert token(0.99, top_p=0.39) == (1, 1.0)
    assert token(0.99, top_p=0.0) == (1, 1.0)
    assert token(0.0, min_p=0.4) == (1, pytest.approx(4 / 9))         # 0.1 / 0.4 < 0.4
    assert token(0.3, temperature=0.0) == (1, 1.0)
    assert token(0.3, temperature=-1.0) == (-1, 0.0) and token(0.3, temperature=math.inf) == (-1, 0.0)
    x = torch.tensor([[-math.inf, math.nan, 1.0, 1.0, 0.0]])
    assert int(ref.sample(x, 0.0 * one)[0]) == 2 and int(ref.sample(x, 0.0 * one, temperature=0 * one)[0]) == 2
    assert int(ref.sample(x, 0.9 * one, top_k=torch.tensor([1]))[0]) == 2
    assert int(ref.sample(torch.full((1, 3), -math.inf), one * 0.5)[0]) == -1
    x = torch.tensor([[1.0, math.inf, 2.0, math.inf]])
    assert int(ref.sample(x, 0.6 * one)[0]) == 3


# ---------------------------------------------------------------- workspaces
@pytest.mark.parametrize("n,i,o", [(130, 8192, 700), (13, 15616, 130), (768, 19968, 3018)])
def test_fc_workspace(n, i, o):
    need = L.cnn_fc_f8_workspace_bytes(n, i, o)
    assert need >= 2 * 4 * n * o and need % (4 * n * o) == 0
    for kw, status in [(dict(work=0, n=need), -4), (dict(work=FAKE, n=need - 1), -4), (dict(work=FAKE + 8, n=need), UNS)]:
        assert _fc(N=n, I=i, O=o, **kw) == status
        assert cnn.cnn_last_error().startswith("fc_f8: workspace")


@pytest.mark.parametrize("n,v", [(1, 40000), (64, 131072), (128, 200000), (1, 2 ** 31 - 1)])
def test_sample_workspace(n, v):
    for t in (F32, BF16):
        need = L.cnn_sample_workspace_bytes(t, n, v)
        assert 0 < need <= n * 80000
        # what a call without cuts needs is what any call needs
        assert _sample(t=t, N=n, V=v, work=FAKE, n=need - 1) == -4
        assert cnn.cnn_last_error().startswith("sample: workspace")
        assert _sample(t=t, N=n, V=v, k=FAKE, work=0, n=need) == -4
