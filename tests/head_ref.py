"""References in 64 bits for the norm, 8-bit floats by block and sampling, and
the bounds their results are held to.  On any device."""
import math

import torch

import experts_ref

F8 = torch.float8_e4m3fn
TOP = 448.0


def blocks_of(cols):
    return -(-cols // 128)


def squares(x, block_rows):
    """x [rows][cols] (float64) as [row blocks][block rows][blocks][128], zeros behind the ends."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, -cols % 128, 0, -rows % block_rows))
    return x.reshape(x.shape[0] // block_rows, block_rows, -1, 128)


def step_f8(v):
    """The step of f8 values at v (float64): 2^(e - 3) from 2^e on, 2^-9 below 2^-6.  (Made of bits: torch.ldexp goes
    through pow, which may be a rounding off and move a midpoint.)"""
    e = (torch.frexp(v)[1].long() - 1).clamp(min=-6)
    return ((e - 3 + 1023) << 52).view(torch.float64)


def nearest_f8(v):
    """The f8 value nearest to v (float64), ties to the even code."""
    step = step_f8(v)
    return (torch.round(v / step) * step).clamp(-TOP, TOP)


def quantize(x, block_rows=1):
    """(values in float64 [rows][cols], scales float32) by the definition: quotients and products rounded to fp32."""
    rows, cols = x.shape
    b = squares(x.double(), block_rows)
    bad = ~torch.isfinite(b).all(3).all(1)
    top = torch.where(bad, 1.0, b.abs().amax((1, 3))).clamp(min=2.0 ** -100)
    most = torch.full_like(top, TOP)
    factor = (most / top).float().double()
    scale = torch.where(bad, math.nan, (top / most).float())
    v = (b * factor[:, None, :, None]).float().double()
    q = torch.where(bad[:, None, :, None], 0.0, nearest_f8(v))
    return q.reshape(-1, q.shape[2] * 128)[:rows, :cols], scale


def spread(scale, rows, cols, block_rows):
    """A scale for every value, float64."""
    return scale.double().repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :cols]


def norm(x, residual, weight, eps):
    """(s in fp32, y in float64)."""
    s = x.float() + residual.float() if residual is not None else x.float()
    d = s.double()
    y = d / (d.square().mean(-1, keepdim=True) + eps).sqrt()
    return s, y * weight.double() if weight is not None else y


def norm_inputs(rows, cols, dtype):
    """x, a residual of its size and weights, whose sums are not numbers of the type: on the CPU, the same ones each time."""
    g = torch.Generator().manual_seed(rows + cols)
    x, r = (torch.randn((rows, cols), generator=g).to(dtype) for _ in range(2))
    return x, r, 1 + 0.2 * torch.randn((cols,), generator=g)


#: y is rounded after the product with 1 / rms (held in 64 bits) and after the weight: two roundings, and a little
NORM_REL = 2.02 * 2.0 ** -24


def assert_norm(y, want, what):
    """y in a wide type."""
    half = 0.0 if y.dtype is torch.float32 else torch.finfo(y.dtype).eps / 2
    tiny = torch.finfo(y.dtype).smallest_normal * torch.finfo(y.dtype).eps
    err = (y.double() - want).abs()
    bound = (NORM_REL * (1 + half) + half) * want.abs() + tiny + 2.0 ** -149
    assert bool((err <= bound).all()), f"{what}: {float((err / bound).max()):.3g} of the bound"


def assert_norm_f8(q, scale, want, what):
    """f8 results: the scale is the block's largest over 448 with one more rounding, every code the nearest one to a
    value off by the results' two roundings, the factor's and its product's."""
    rows, cols = want.shape
    top = squares(want, 1).abs().amax((1, 3)).clamp(min=2.0 ** -100)
    assert scale.shape == top.shape and q.shape == want.shape
    off = (scale.double() - top / TOP).abs()
    assert bool((off <= (NORM_REL + 2.0 ** -24) * top / TOP * 1.01).all()), what
    v = want * spread(TOP / top, rows, cols, 1)
    # top and value are off by NORM_REL each, the factor and the product by 2^-24 each
    slack = (2 * NORM_REL + 2 * 2.0 ** -24) * 1.01 * v.abs()
    near = (v.abs() + slack).clamp(max=TOP)
    err = (q.double() - v).abs()
    assert bool((err <= step_f8(near) / 2 + slack).all()), what


def product(x, xs, w, ws, b, relu):
    """(x w^T + b, sum of magnitudes), float64, of f8 values with scales."""
    (n, i), o = x.shape, w.shape[0]
    a = x.double() * spread(xs, n, i, 1)
    c = w.double() * spread(ws, o, i, 128)
    y, s = a @ c.T, a.abs() @ c.abs().T
    if b is not None:
        y, s = y + b.double(), s + b.double().abs()
    if relu:
        y = torch.where(y > 0, y, 0.0)
    return y, s


def steps(i):
    """Additions and roundings of a sum of i products: those of every block, and for each block the scales' product, the
    product with it, the addition; and those of parts that are joined."""
    return i + 3 * blocks_of(i) + 32


def assert_product(got, want, s, i, what):
    """A product's results against the float64 ones.

    fp32 results: every product is exact and added in fp32, so that experts_ref's bound holds, a step of 2^-23 of the sum
    of magnitudes S for every addition and rounding.  16-bit results are those rounded, which test_gpu_f8_ways holds
    them to by equality; the bounds here are wider: they would allow for products added by eights in steps of 2^-13 of
    the power of two at or below the largest of them: 8 steps a group, no more than 2^-10 of the group's S, and of all
    S in sum.  The groups' errors would be independent, so that their 2-norm is within 2^-10 S / sqrt(groups) for S
    spread over them; twice that is allowed."""
    if got.dtype is torch.float32:
        experts_ref.assert_product(got, want, s, steps(i), what)
        return
    half = torch.finfo(got.dtype).eps / 2
    tiny = torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps
    err = (got.double() - want).abs()
    assert bool(torch.isfinite(err).all()), f"{what}: not finite"
    bound = half * want.abs() + (2.0 ** -10 + steps(i) * 2.0 ** -23) * s * (1 + half) + tiny
    assert bool((err <= bound).all()), f"{what}: {float((err / bound).max()):.3g} of its bound"
    norm, groups = float(err.norm()), -(-i // 8)
    most = half * float(want.norm()) + (2.0 ** -9 / math.sqrt(groups) + 2.0 ** -22) * float(s.norm()) + tiny * math.sqrt(err.numel())
    assert norm <= most, f"{what}: error norm {norm:.3g}, bound {most:.3g}"


def random_f8(shape, gen, size=100.0):
    return (size * torch.randn(shape, generator=gen, device=gen.device)).clamp(-TOP, TOP).to(F8)


def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """(token, probability, distance) by sorting in float64, row by row.  distance: how near to another result the row
    is: the least distance of a sum from the border that it is compared with, as a share of all of them, and of a weight
    from min_p."""
    n, v = logits.shape
    x = logits.double().cpu()
    par = [None if t is None else t.double().cpu() for t in (u, temperature, top_k, top_p, min_p)]
    tokens, probs, far = [], [], []
    for r in range(n):
        row = x[r]
        draw = float(par[0][r])
        temp, k, p, least = (d if t is None else float(t[r]) for t, d in zip(par[1:], (1.0, 0.0, 1.0, 0.0)))
        live = torch.nonzero(row > -math.inf).flatten()  # not NaN
        if not len(live) or not (0 <= temp < math.inf) or any(math.isnan(t) for t in (draw, p, least)):
            tokens.append(-1), probs.append(0.0), far.append(1.0)
            continue
        top = float(row[live].max())
        if top == math.inf:
            live = live[row[live] == math.inf]
        order = live[torch.argsort(row[live], descending=True, stable=True)]
        if temp == 0:
            tokens.append(int(order[0])), probs.append(1.0), far.append(1.0)
            continue
        w = torch.exp((row[order] - top) / temp) if top < math.inf else torch.ones(len(order), dtype=torch.float64)
        near = 1.0
        if k > 0:
            order, w = order[:int(k)], w[:int(k)]
        if p < 1:
            sums = w.cumsum(0)
            border = p * float(sums[-1])
            keep = (sums - w) < border
            keep[0] = True
            if p > 0:
                near = min(near, float((sums[:-1] - border).abs().min()) / float(sums[-1])) if len(w) > 1 else near
            order, w = order[keep], w[keep]
        if least > 0:
            keep = w >= least
            keep[0] = True
            other = w[w < 1]
            near = min(near, float((other - least).abs().min())) if len(other) else near
            order, w = order[keep], w[keep]
        by = torch.argsort(order)
        order, w = order[by], w[by]
        sums = w.cumsum(0)
        t = min(max(draw, 0.0), 1 - 2.0 ** -40) * float(sums[-1])
        at = int(torch.searchsorted(sums, t, right=True))
        near = min(near, float((sums[:-1] - t).abs().min()) / float(sums[-1])) if len(w) > 1 and 0 < draw < 1 else near
        tokens.append(int(order[at])), probs.append(float(w[at] / sums[-1])), far.append(near)
    return (torch.tensor(tokens, dtype=torch.int32), torch.tensor(probs, dtype=torch.float64),
            torch.tensor(far, dtype=torch.float64))


def assert_sample(got, want, what):
    """Tokens are equal, but for rows that stand within 1e-9 of another result: weights are held to 2^-43 of the
    largest (V up to 2^20) and the reference's sums to 2^-53 of all, so that sums of 2^20 weights are off by less.
    Probabilities: one rounding to fp32, and 1e-6 for weights that are held to few bits."""
    token, prob = got[0].cpu(), got[1].double().cpu()
    same = token == want[0]
    clear = want[2] > 1e-9
    assert bool((same | ~clear).all()), (what, token[~same & clear], want[0][~same & clear])
    assert int((~clear).sum()) <= max(1, len(token) // 100), what
    err = (prob - want[1]).abs()
    assert bool((err[same] <= 2.0 ** -24 * want[1][same] + 1e-6 * want[1][same] + 2.0 ** -40).all()), what
