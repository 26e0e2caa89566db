"""The operators behind a network's body together, as a program that answers runs them (GPU): RMS norm to 8-bit floats,
two fully connected layers on them, the norm with the residual, the layer that gives the logits, the token.  Every
stage is compared with its reference in 64 bits on what the stage before gave (``head_ref``)."""
import math

import pytest
import torch

import head_ref as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
IDS = ["f32", "bf16", "f16"]
EPS = 1e-5


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(shape, g, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


class Head:
    """t tokens of d values, a layer of f, v logits; weights in 8 bits."""

    def __init__(self, gpu, dtype, t, d, f, v, seed):
        g = gen(seed)
        self.gpu, self.dtype = gpu, dtype
        self.x, self.r = randn((t, d), g, dtype), randn((t, d), g, dtype)
        self.norms = [1 + 0.1 * randn((d,), g) for _ in range(2)]
        self.w = [gpu.cnn_f8_quantize(randn((o, i), g) / math.sqrt(i), 128) for o, i in ((f, d), (d, f), (v, d))]
        self.b = [0.1 * randn((f,), g), None, None]
        self.u = torch.rand((t,), generator=g, device="cuda")
        self.cuts = {"temperature": torch.full((t,), 0.3, device="cuda"),
                     "top_k": torch.full((t,), 40, device="cuda", dtype=torch.int32),
                     "top_p": torch.full((t,), 0.9, device="cuda"), "min_p": torch.full((t,), 0.01, device="cuda")}

    def stages(self, x=None, u=None, stream=None):
        gpu, kw = self.gpu, {"stream": stream}
        x, u = self.x if x is None else x, self.u if u is None else u
        q1, s1, sum1 = gpu.cnn_rms_norm_fwd(x, self.norms[0], self.r, EPS, f8=True, **kw)
        h = gpu.cnn_fc_f8_fwd(q1, s1, *self.w[0], self.b[0], True, y_dtype=self.dtype, **kw)
        q2, s2 = gpu.cnn_f8_quantize(h, **kw)
        y = gpu.cnn_fc_f8_fwd(q2, s2, *self.w[1], y_dtype=self.dtype, **kw)
        q3, s3, sum3 = gpu.cnn_rms_norm_fwd(y, self.norms[1], sum1, EPS, f8=True, **kw)
        logits = gpu.cnn_fc_f8_fwd(q3, s3, *self.w[2], **kw)
        return x, (q1, s1, sum1), h, (q2, s2), y, (q3, s3, sum3), logits, gpu.cnn_sample_fwd(logits, u, **self.cuts, **kw)

    def __call__(self, *a, **kw):
        """What a program keeps: the residual, the logits, the tokens and their probabilities."""
        *_, (_, _, total), logits, (token, prob) = self.stages(*a, **kw)
        return total, logits, token, prob


def same(got, want):
    return all(torch.equal(a, b) for a, b in zip(got, want))


SIZES = [(1, 128, 256, 1000), (3, 512, 1280, 40000), (5, 200, 333, 517), (70, 384, 1024, 4001), (300, 1000, 640, 999),
         (1100, 256, 1536, 2000)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("t,d,f,v", SIZES)
def test_head(gpu, t, d, f, v, dtype):
    m = Head(gpu, dtype, t, d, f, v, t + d)
    x, n1, h, q2, y, n3, logits, token = m.stages()
    what = f"{t} {d} {f} {v} {dtype}"
    for (q, s, total), a, r, w in ((n1, x, m.r, m.norms[0]), (n3, y, n1[2], m.norms[1])):
        wide, want = ref.norm(a, r, w, EPS)
        assert torch.equal(total, wide.to(dtype))
        ref.assert_norm_f8(q, s, want, what)
    assert torch.equal(q2[0].double(), ref.quantize(h)[0]) and torch.equal(q2[1], ref.quantize(h)[1])
    for got, (q, s), k, relu in ((h, n1[:2], 0, True), (y, q2, 1, False), (logits, n3[:2], 2, False)):
        want, size = ref.product(q, s, *m.w[k], m.b[k], relu)
        ref.assert_product(got, want, size, q.shape[1], what)
    few = slice(0, 50)
    ref.assert_sample([k[few] for k in token], ref.sample(logits[few], m.u[few], **{k: c[few] for k, c in m.cuts.items()}), what)
    assert bool((token[0] >= 0).all()) and bool((token[0] < v).all())


def test_head_padded_batch(gpu):
    """Rows that pad a batch, NaN among them, change nothing of the others'."""
    m = Head(gpu, torch.bfloat16, 40, 512, 768, 3000, 3)
    want = m()
    for pad in (math.nan, math.inf, 0.0):
        x = m.x.clone()
        x[7], x[33:] = pad, pad
        got = m(x)
        live = torch.ones(40, dtype=torch.bool, device="cuda")
        live[7], live[33:] = False, False
        assert same([k[live] for k in got], [k[live] for k in want])
        if math.isnan(pad) or math.isinf(pad):
            assert bool((got[2][~live] == -1).all())


@pytest.mark.parametrize("t", [3, 150])
def test_head_captured(gpu, t):
    """Captured and replayed with new inputs in the same buffers, with eager work of its own between; two graphs
    of it share nothing.  40000 logits: 3 rows are split over workgroups."""
    m = Head(gpu, torch.bfloat16, t, 512, 1280, 40000, 5)
    m()
    torch.cuda.synchronize()
    x, u = m.x.clone(), m.u.clone()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = m(x, u)
        graphs.append((g, y))
    for i in range(3):
        r = gen(60 + i)
        x.copy_(randn(x.shape, r, x.dtype))
        u.copy_(torch.rand(u.shape, generator=r, device="cuda"))
        eager = m(x, u)
        for _, y in graphs:
            for k in y:
                k.fill_(-7)
        for g, _ in graphs:
            g.replay()
        between = m()
        torch.cuda.synchronize()
        for _, y in graphs:
            assert same(y, eager), i
        assert bool((between[2] >= 0).all())


@pytest.mark.parametrize("t", [2, 200])
def test_head_on_another_stream(gpu, t):
    """Two passes at once on streams of their own, given as an argument and as the current stream."""
    one = Head(gpu, torch.bfloat16, t, 512, 1280, 40000, 7)
    two = Head(gpu, torch.float32, t, 384, 640, 5000, 8)
    want = one(), two()
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        got_one = one(stream=a)
        with torch.cuda.stream(b):
            got_two = two()
        raw = two(stream=a.cuda_stream)
        torch.cuda.synchronize()
        assert same(got_one, want[0]) and same(got_two, want[1]) and same(raw, want[1])


# ---------------------------------------------------------------- the product's ways
# Sizes at which each of them is taken: by rows of 16 x 32; tiles of 64 x 128, 128 x 128, 128 x 256 and 256 x 256 tokens x
# outputs, whole and with the reduction split, from vectors and through registers.
WAYS = [(3, 130, 9000), (651, 128, 1166), (13, 15616, 130), (5499, 128, 1040), (3161, 15744, 3), (3536, 128, 1676),
        (2114, 20736, 422), (6535, 128, 1797), (768, 19968, 3018), (1214, 58752, 1774), (759, 246, 1054), (15, 16253, 130),
        (3992, 47, 777), (459, 2171, 1467), (4171, 128, 386), (64, 9216, 4096), (12, 24543, 1), (20, 16145, 2), (335, 1905, 1355),
        (807, 2211, 423), (491, 2226, 958), (1688, 1362, 2688), (16, 32631, 5), (1631, 8704, 1159), (1805, 20352, 2259),
        (587, 5760, 3442), (885, 250, 646), (768, 119, 1090)]


def operands(n, i, o, seed):
    g = gen(seed)
    x, w, nb = ref.random_f8((n, i), g), ref.random_f8((o, i), g), ref.blocks_of(i)
    return (x, torch.exp(0.5 * randn((n, nb), g)) / 100, w, torch.exp(0.5 * randn((ref.blocks_of(o), nb), g)) / (100 * math.sqrt(i)),
            0.1 * randn((o,), g))


@pytest.mark.parametrize("n,i,o", WAYS)
def test_product_every_way(gpu, n, i, o):
    x, xs, w, ws, b = operands(n, i, o, n + o)
    want, s = ref.product(x, xs, w, ws, b, False)
    for dtype in (torch.float32, torch.bfloat16):
        room = torch.full((n * o + 128,), 7.0, dtype=dtype, device="cuda")
        y = gpu.cnn_fc_f8_fwd(x, xs, w, ws, b, y=room[64:64 + n * o].view(n, o))
        ref.assert_product(y, want, s, i, f"{n}x{i}x{o} {dtype}")
        assert bool((room[:64] == 7).all()) and bool((room[64 + n * o:] == 7).all())


@pytest.mark.parametrize("n,i,o", [(3, 130, 9000), (651, 128, 1166), (3536, 128, 1676), (6535, 128, 1797), (768, 19968, 3018)])
def test_product_every_way_at_odd_addresses(gpu, n, i, o):
    """Operands at bytes that no vector begins at, results at their type's second place; among NaN."""
    x, xs, w, ws, b = operands(n, i, o, n + i)
    want, s = ref.product(x, xs, w, ws, b, False)

    def moved(v, by):
        room = torch.full((v.numel() + 64,), 0x7f, dtype=torch.uint8, device="cuda").view(ref.F8)
        room[by:by + v.numel()].copy_(v.reshape(-1))
        return room[by:by + v.numel()].view(v.shape)
    y = torch.empty((n * o + 1,), dtype=torch.float16, device="cuda")[1:].view(n, o)
    gpu.cnn_fc_f8_fwd(moved(x, 3), xs, moved(w, 17), ws, b, y=y)
    ref.assert_product(y, want, s, i, f"{n}x{i}x{o}")


@pytest.mark.parametrize("n,o", [(600, 1200), (2305, 776), (4000, 1100), (3400, 2440)])
def test_product_numbers_of_blocks(gpu, n, o):
    """Reductions of one block, of as many as there are buffers, of a few more."""
    for blocks in (*range(1, 10), 13):
        x, xs, w, ws, b = operands(n, 128 * blocks, o, n + blocks)
        want, s = ref.product(x, xs, w, ws, b, False)
        for dtype in (torch.float32, torch.float16):
            y = gpu.cnn_fc_f8_fwd(x, xs, w, ws, b, y_dtype=dtype)
            ref.assert_product(y, want, s, 128 * blocks, f"{n}x{128 * blocks}x{o} {dtype}")
            for _ in range(3):
                assert torch.equal(y, gpu.cnn_fc_f8_fwd(x, xs, w, ws, b, y_dtype=dtype))
