"""References in 64 bits for the operators on microscaled 4-bit values and on
groups of rows, and the bounds their results are held to.

Products: a sum of n products, exact or rounded to fp32 in any order, is off
by at most n steps of 2^-23 of S = sum |x w| + |b| (a step for every addition,
whether the matrix cores round or cut), and rounding the result once to type T
adds eps(T)/2 of it.  That bound is loose for long sums, so the error's 2-norm
is held too: errors of single additions are independent, so that it grows
with sqrt(n); twice sqrt(n + 16) 2^-24 of the 2-norm of S over sqrt(n) (the size
of a sum of independent terms), plus the rounding of the result.
"""
import math

import torch

CODES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def blocks_of(cols):
    return -(-cols // 32)


def two_to(e):
    """2^e in float64 for whole e, exactly (pow may be a rounding off, which would move a midpoint)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def quantize(x):
    """(q, scale) of x [rows][cols], by the definition: a search over the eight magnitudes."""
    rows, cols = x.shape
    b = torch.nn.functional.pad(x.double(), (0, -cols % 32)).reshape(rows, -1, 32)
    top = b.abs().amax(-1)
    bad = ~torch.isfinite(b).all(-1)
    fine = torch.where(bad, 1.0, top).clamp(min=2.0 ** -149)
    _, e = torch.frexp(fine)                      # top = m 2^e, 0.5 <= m < 1
    s = (e - 1 - 2 + 127).clamp(min=0)
    a = b.abs() / two_to(s - 127).unsqueeze(-1)
    table = torch.tensor(CODES, dtype=torch.float64, device=x.device)
    dist = (a.unsqueeze(-1) - table).abs()
    # of two as near, the even code
    preference = torch.tensor([0, 4, 1, 5, 2, 6, 3, 7], device=x.device)
    code = torch.where(dist == dist.amin(-1, keepdim=True), preference, 8).argmin(-1)
    code = code + 8 * torch.signbit(b)
    code = torch.where(bad.unsqueeze(-1), 0, code).to(torch.uint8).reshape(rows, -1)
    q = code[:, 0::2] | (code[:, 1::2] << 4)
    return q, torch.where(bad, 255, s).to(torch.uint8)


def values(q, scale, cols):
    """The values of mx4 rows, float64."""
    table = torch.tensor(CODES + tuple(-c for c in CODES), dtype=torch.float64, device=q.device)
    v = table[torch.stack([q & 15, q >> 4], -1).flatten(-2).long()]
    s = two_to(scale.long() - 127)
    s = torch.where(scale == 255, float("nan"), s)
    return (v * s.repeat_interleave(32, dim=-1))[..., :cols]


def random_mx4(lead, cols, gen, spread=3):
    """Random mx4 rows (zeros behind the last column), scales around 1 / sqrt(cols)."""
    nb = blocks_of(cols)
    q = torch.randint(0, 256, lead + (nb * 16,), generator=gen, device=gen.device, dtype=torch.uint8)
    at = 2 * torch.arange(nb * 16, device=gen.device)
    q &= (0x0F * (at < cols) + 0xF0 * (at + 1 < cols)).to(torch.uint8)
    mid = 127 - int(round(math.log2(8 * cols) / 2))
    scale = torch.randint(mid - spread, mid + spread, lead + (nb,), generator=gen, device=gen.device, dtype=torch.uint8)
    return q, scale


def product(x, w, b, relu):
    """(x w^T + b, sum of magnitudes), float64."""
    y = x.double() @ w.double().T
    s = x.double().abs() @ w.double().abs().T
    if b is not None:
        y = y + b.double()
        s = s + b.double().abs()
    if relu:
        y = torch.where(y > 0, y, 0.0)
    return y, s


def assert_product(got, ref, s, n, what):
    """got (any wide type) against the float64 result; n: products a sum."""
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    if ref.numel() == 0:
        return
    half = torch.finfo(got.dtype).eps / 2
    tiny = torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps  # a step of subnormal results
    err = (got.double() - ref).abs()
    assert bool(torch.isfinite(err).all()), f"{what}: not finite"
    bound = half * ref.abs() + (n + 2) * 2.0 ** -23 * s * (1 + half) + tiny
    worst = float((err / bound).max())
    assert worst <= 1, f"{what}: error {worst:.3g} of its bound"
    norm = float(err.norm())
    most = half * float(ref.norm()) + 2 * math.sqrt(n + 16) * 2.0 ** -24 * float(s.norm()) / math.sqrt(n) + tiny * math.sqrt(err.numel())
    assert norm <= most, f"{what}: error norm {norm:.3g}, bound {most:.3g}"


def route(logits, k, renorm):
    """The router's outputs by sorting (expert, weight in float64, rows, offsets, slot)."""
    T, E = logits.shape
    v = logits.double()
    may = v > -math.inf                          # false for NaN
    # stable, so that equal logits stay in the order of the experts; +0 and -0 are equal
    key = torch.where(may, v, -math.inf)
    order = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :k]
    there = may.gather(1, order)
    top = torch.where(may, v, -math.inf).amax(1, keepdim=True)
    p = torch.where(may, torch.exp(v - top), 0.0)
    chosen = torch.where(there, p.gather(1, order), 0.0)
    weight = chosen / (chosen if renorm else p).sum(1, keepdim=True)
    weight = torch.where(there, weight, 0.0)
    expert = torch.where(there, order, -1).to(torch.int32)
    flat = expert.reshape(-1)
    at = torch.argsort(torch.where(flat < 0, E, flat), stable=True)
    n = int((flat >= 0).sum())
    rows = torch.full((T * k,), -1, dtype=torch.int32, device=logits.device)
    rows[:n] = (at[:n] // k).to(torch.int32)
    slot = torch.full((T * k,), -1, dtype=torch.int32, device=logits.device)
    slot[at[:n]] = torch.arange(n, dtype=torch.int32, device=logits.device)
    counts = torch.bincount(flat[flat >= 0].long(), minlength=E)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
    return expert, weight, rows, offsets, slot.reshape(T, k)
