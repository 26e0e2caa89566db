"""Sampling with temperature, top-k, top-p and min-p (GPU), against a reference
that sorts in 64 bits (``head_ref``)."""
import math

import pytest
import torch

import head_ref as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
IDS = ["f32", "bf16", "f16"]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rand(n, g):
    return torch.rand((n,), generator=g, device="cuda")


def logits(n, v, g, dtype, size=2.0):
    x = size * torch.randn((n, v), generator=g, device="cuda")
    at = torch.randint(0, v, (n, min(v, 16)), generator=g, device="cuda")
    x.scatter_add_(1, at, 7 * torch.rand(at.shape, generator=g, device="cuda"))
    return x.to(dtype)


def parameters(n, v, g, rules):
    kw = {}
    if "t" in rules:
        kw["temperature"] = 0.4 + rand(n, g)
    if "k" in rules:
        kw["top_k"] = torch.randint(0, max(2, min(v + 2, 300)), (n,), generator=g, device="cuda", dtype=torch.int32)
    if "p" in rules:
        kw["top_p"] = 0.2 + 0.9 * rand(n, g)
    if "m" in rules:
        kw["min_p"] = 0.2 * rand(n, g)
    return kw


SIZES = [(1, 1), (2, 2), (5, 7), (3, 64), (9, 1000), (2, 4096), (2, 4097), (1, 32768), (3, 50021), (2, 131072), (300, 50)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("rules", ["", "t", "tk", "tp", "tm", "kp", "tkpm"])
@pytest.mark.parametrize("n,v", SIZES)
def test_sample(gpu, n, v, rules, dtype):
    g = gen(n + v)
    x, u, kw = logits(n, v, g, dtype), rand(n, g), parameters(n, v, g, rules)
    ref.assert_sample(gpu.cnn_sample_fwd(x, u, **kw), ref.sample(x, u, **kw), f"{n}x{v} {rules} {dtype}")


@pytest.mark.parametrize("rules", ["t", "tk", "tp", "tkpm"])
def test_sample_every_place(gpu, rules):
    """One row's distribution walked through: u from 0 to 1 in 257 rows of the same logits."""
    g = gen(3)
    n, v = 257, 700
    x = logits(1, v, g, torch.float32).repeat(n, 1)
    kw = {k: t[:1].repeat(n) for k, t in dict(temperature=0.8 + rand(1, g), top_k=torch.full((1,), 40, device="cuda", dtype=torch.int32),
                                              top_p=torch.full((1,), 0.9, device="cuda"),
                                              min_p=torch.full((1,), 0.02, device="cuda")).items() if k[0] in rules or k[-1] in rules}
    u = torch.linspace(0, 1, n, device="cuda")
    got = gpu.cnn_sample_fwd(x, u, **kw)
    ref.assert_sample(got, ref.sample(x, u, **kw), rules)
    assert bool((got[0][1:] >= got[0][:-1]).all())


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("v", [40, 3000, 9000, 70000])
def test_sample_ties(gpu, v, dtype):
    """Rows with few different logits, so that borders fall among equals: the lowest tokens are kept.  More of them than
    fit the list that a row is worked on in."""
    g = gen(v)
    n = 24
    x = torch.randint(-2, 3, (n, v), generator=g, device="cuda").to(dtype)
    x[0] = 1.0
    x[1] = 0.0
    x[1, ::2] = -0.0
    u = rand(n, g)
    k = torch.randint(1, v + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
    for kw in ({}, {"top_k": k}, {"top_p": 0.05 + 0.94 * rand(n, g)}, {"top_k": k, "top_p": 0.05 + 0.94 * rand(n, g)},
               {"top_k": k, "min_p": rand(n, g)}, {"min_p": torch.ones((n,), device="cuda")},
               {"temperature": 0.02 + 0.1 * rand(n, g), "top_k": k, "top_p": 0.99 + 0.009 * rand(n, g)}):
        ref.assert_sample(gpu.cnn_sample_fwd(x, u, **kw), ref.sample(x, u, **kw), f"{v} {dtype} {list(kw)}")


@pytest.mark.parametrize("v", [3000, 30000, 140000])
def test_sample_flat_rows(gpu, v):
    """Logits that lie close together or far apart: one bin of weights or all of them, more tokens than the list holds."""
    g = gen(v + 1)
    n = 6
    base = torch.randn((n, v), generator=g, device="cuda")
    for size in (1e-6, 1e-3, 0.05, 1.0, 30.0):
        for shift in (0.0, 100.0):
            x, u = size * base + shift, rand(n, g)
            kw = {"top_k": torch.tensor([0, 5, v // 2, v - 1, v, 3 * v], device="cuda", dtype=torch.int32),
                  "top_p": torch.tensor([0.5, 1.0, 0.7, 0.999, 0.3, 0.95], device="cuda")}
            ref.assert_sample(gpu.cnn_sample_fwd(x, u, **kw), ref.sample(x, u, **kw), f"{v} {size} {shift}")


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("v", [5, 1000, 40000])
def test_sample_masks(gpu, v, dtype):
    """Rows that are masked in part, wholly, by the type's lowest value, with NaN and infinities."""
    g = gen(v + 2)
    x = logits(10, v, g, dtype)
    low = torch.finfo(dtype).min
    x[0] = -math.inf
    x[1, : v - 1] = -math.inf
    x[2] = math.nan
    x[3, 1:] = math.nan
    x[4] = low
    x[5, : v - 2] = low
    x[6, 1], x[6, 3] = math.inf, math.inf
    x[7, ::2] = -math.inf
    x[7, 1] = math.nan
    x[8] = torch.finfo(dtype).max
    x[8, 2] = low
    x[9, 0] = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    u = rand(10, g)
    for kw in ({}, {"top_k": torch.full((10,), 3, device="cuda", dtype=torch.int32)}, {"top_p": torch.full((10,), 0.8, device="cuda")},
               {"min_p": torch.full((10,), 0.3, device="cuda")}, {"temperature": torch.zeros((10,), device="cuda")},
               {"temperature": torch.full((10,), 1e-3, device="cuda"), "top_p": torch.full((10,), 0.8, device="cuda")}):
        got = gpu.cnn_sample_fwd(x, u, **kw)
        ref.assert_sample(got, ref.sample(x, u, **kw), f"{v} {dtype} {list(kw)}")
        assert int(got[0][0]) == -1 and int(got[0][1]) == v - 1 and int(got[0][2]) == -1 and int(got[0][3]) == 0
        assert int(got[0][6]) in (1, 3)


def test_sample_parameters_at_their_ends(gpu):
    """Each parameter at and beyond its range, with the token and probability that the definition gives."""
    nan, inf = math.nan, math.inf
    x = torch.log(torch.tensor([0.1, 0.4, 0.2, 0.3], device="cuda"))
    cases = [  # u, temperature, k, p, m, token, prob
        (0.5, 1.0, 0, 1.0, 0.0, None, None), (0.0, 1.0, 0, 1.0, 0.0, 0, 0.1), (-3.0, 1.0, 0, 1.0, 0.0, 0, 0.1),
        (1.0, 1.0, 0, 1.0, 0.0, 3, 0.3), (7.0, 1.0, 0, 1.0, 0.0, 3, 0.3), (inf, 1.0, 0, 1.0, 0.0, 3, 0.3), (nan, 1.0, 0, 1.0, 0.0, -1, 0.0),
        (0.9, 0.0, 0, 1.0, 0.0, 1, 1.0), (0.9, -0.0, 3, 0.5, 0.1, 1, 1.0), (0.9, -1.0, 0, 1.0, 0.0, -1, 0.0), (0.9, nan, 0, 1.0, 0.0, -1, 0.0),
        (0.9, inf, 0, 1.0, 0.0, -1, 0.0), (0.9, 1e-30, 0, 1.0, 0.0, 1, 1.0), (0.9, 1e-44, 0, 0.5, 0.0, 1, 1.0), (0.9, 1e38, 0, 1.0, 0.0, 3, 0.25),
        (0.1, 3.4e38, 2, 0.9, 0.0, 1, 0.5),
        (0.9, 1.0, 1, 1.0, 0.0, 1, 1.0), (0.9, 1.0, -5, 1.0, 0.0, 3, 0.3), (0.9, 1.0, 2**31 - 1, 1.0, 0.0, 3, 0.3), (0.0, 1.0, 3, 1.0, 0.0, 1, 4 / 9),
        (0.9, 1.0, 0, 0.0, 0.0, 1, 1.0), (0.9, 1.0, 0, -1.0, 0.0, 1, 1.0), (0.9, 1.0, 0, nan, 0.0, -1, 0.0), (0.9, 1.0, 0, 5.0, 0.0, 3, 0.3),
        (0.9, 1.0, 0, 1e-30, 0.0, 1, 1.0), (0.9, 1.0, 0, inf, 0.0, 3, 0.3),
        (0.9, 1.0, 0, 1.0, 1.0, 1, 1.0), (0.9, 1.0, 0, 1.0, 2.0, 1, 1.0), (0.9, 1.0, 0, 1.0, nan, -1, 0.0), (0.9, 1.0, 0, 1.0, -1.0, 3, 0.3),
        (0.0, 1.0, 0, 1.0, 0.3, 1, 4 / 9), (0.9, 1.0, 0, 1.0, 1e-30, 3, 0.3), (0.9, 1.0, 0, 1.0, inf, 1, 1.0),
    ]
    n = len(cases)
    t = [torch.tensor([c[j] for c in cases], device="cuda", dtype=torch.int32 if j == 2 else torch.float32) for j in range(5)]
    for wide in (4, 5000, 40000):
        rows = torch.full((n, wide), -math.inf, device="cuda")
        rows[:, :4] = x
        token, prob = gpu.cnn_sample_fwd(rows, *t)
        for j, c in enumerate(cases):
            if c[5] is not None:
                assert int(token[j]) == c[5], (wide, c, int(token[j]))
                assert abs(float(prob[j]) - c[6]) <= 1e-6, (wide, c, float(prob[j]))


def test_sample_follows_the_distribution(gpu):
    """Counts of 20000 draws against their expectation, each within 5 standard deviations."""
    g = gen(8)
    n, v = 20000, 30
    x = (1.5 * torch.randn((1, v), generator=g, device="cuda")).repeat(n, 1)
    token, prob = gpu.cnn_sample_fwd(x, rand(n, g))
    p = torch.softmax(x[0].double(), 0)
    count = torch.bincount(token.long(), minlength=v).double()
    assert bool(((count - n * p).abs() <= 5 * (n * p * (1 - p)).sqrt() + 1).all())
    assert bool(((prob.double() - p[token.long()]).abs() <= 1e-6).all())


def test_sample_is_the_same_every_time_and_by_row(gpu):
    """A row's token does not depend on the rows beside it, nor on the call."""
    g = gen(9)
    n, v = 40, 20000
    x, u, kw = logits(n, v, g, torch.bfloat16), rand(n, g), parameters(n, v, g, "tkpm")
    token, prob = gpu.cnn_sample_fwd(x, u, **kw)
    for _ in range(2):
        again = gpu.cnn_sample_fwd(x, u, **kw)
        assert torch.equal(token, again[0]) and torch.equal(prob, again[1])
    for r in (0, 7, 39):
        one = gpu.cnn_sample_fwd(x[r:r + 1], u[r:r + 1], **{k: t[r:r + 1] for k, t in kw.items()})
        assert torch.equal(one[0], token[r:r + 1]) and torch.equal(one[1], prob[r:r + 1])


def test_sample_at_any_address(gpu):
    """Rows of an odd length, which begin at any multiple of their type, among NaN and infinities that are not theirs."""
    g = gen(10)
    for dtype in TYPES:
        for v in (333, 9001):
            x, u = logits(4, v, g, dtype), rand(4, g)
            room = torch.full((4 * v + 9,), math.inf, dtype=dtype, device="cuda")
            at = room[3:3 + 4 * v].view(4, v)
            at.copy_(x)
            k = torch.full((4,), 20, device="cuda", dtype=torch.int32)
            for kw in ({}, {"top_k": k}):
                a, b = gpu.cnn_sample_fwd(at, u, **kw), gpu.cnn_sample_fwd(x, u, **kw)
                assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_sample_refuses_and_empty(gpu):
    x, u = torch.zeros((4, 50), device="cuda"), torch.zeros((4,), device="cuda")
    token, prob = gpu.cnn_sample_fwd(x[:0], u[:0])
    assert token.shape == (0,) and prob.shape == (0,) and token.dtype is torch.int32 and prob.dtype is torch.float32
    k = torch.ones((4,), device="cuda", dtype=torch.int32)
    for call, error in [
        (lambda: gpu.cnn_sample_fwd(x.double(), u), TypeError),
        (lambda: gpu.cnn_sample_fwd(x[0], u), ValueError),
        (lambda: gpu.cnn_sample_fwd(x.T, u), TypeError),
        (lambda: gpu.cnn_sample_fwd(x, None), TypeError),
        (lambda: gpu.cnn_sample_fwd(x, u[:3]), ValueError),
        (lambda: gpu.cnn_sample_fwd(x, u.double()), TypeError),
        (lambda: gpu.cnn_sample_fwd(x, u, u.half()), TypeError),
        (lambda: gpu.cnn_sample_fwd(x, u, top_k=u), TypeError),
        (lambda: gpu.cnn_sample_fwd(x, u, top_k=k.long()), TypeError),
        (lambda: gpu.cnn_sample_fwd(x, u, top_p=0.9), TypeError),
        (lambda: gpu.cnn_sample_fwd(x, u, min_p=u.cpu()), TypeError),
        (lambda: gpu.cnn_sample_fwd(x[:, :0].contiguous(), u), gpu.CnnError),
    ]:
        with pytest.raises(error):
            call()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("v", [20001, 45000, 70001])
def test_sample_however_rows_are_shared_out(gpu, v, dtype):
    """One row, few or many: its work goes to one workgroup or to several, its token and probability are the same."""
    g = gen(v)
    n = 140
    x, u, kw = logits(n, v, g, dtype), rand(n, g), parameters(n, v, g, "tkpm")
    for keys in ((), ("temperature", "min_p"), ("top_p",), tuple(kw)):
        some = {k: kw[k] for k in keys}
        token, prob = gpu.cnn_sample_fwd(x, u, **some)
        for rows in (slice(0, 1), slice(3, 60)):
            part = gpu.cnn_sample_fwd(x[rows], u[rows], **{k: t[rows] for k, t in some.items()})
            assert torch.equal(part[0], token[rows]) and torch.equal(part[1], prob[rows])
