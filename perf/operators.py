"""The operators of a served mixture-of-experts block and of weights held in 4 bits, and the calls they are measured by.

Each case is one call (quantisation: there and back) that a program makes
through the Python binding of libcnn, with its plain form in elementary torch
operations.  Microscaled 4-bit values ("mx4") are blocks of 32 along a row:
a byte holds two values of 1 sign, 2 exponent and 1 mantissa bits, low half
first, and a byte per block its power-of-two scale, biased by 127.  Wide types
are those of the activations; biases and routing weights are fp32.
"""
from __future__ import annotations

import math

import torch

own = False  # True: run() calls the library's kernels; False: their plain forms

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2, "mx4": 17 / 32}


def _quant(rows, cols, dtype):
    return {"op": "quantize", "rows": rows, "cols": cols, "dtype": dtype}


def _fc(n, i, o, dtype, x4, relu):
    """x4: the activations are brought to mx4 too, in the call."""
    return {"op": "fc_mx4", "n": n, "i": i, "o": o, "dtype": dtype, "x4": x4, "relu": relu}


def _grouped(tokens, experts, k, i, o, dtype, w4, relu):
    """w4: the experts' weights are held in mx4."""
    return {"op": "grouped", "tokens": tokens, "experts": experts, "k": k, "i": i, "o": o, "dtype": dtype,
            "w4": w4, "relu": relu}


def _route(tokens, experts, k, dtype, renorm):
    return {"op": "route", "tokens": tokens, "experts": experts, "k": k, "dtype": dtype, "renorm": renorm}


def _combine(tokens, k, d, dtype):
    return {"op": "combine", "tokens": tokens, "k": k, "d": d, "dtype": dtype}


def listed():
    cases = {
        # the activations of a batch of 64 before a product of two 4-bit operands
        "quantize_act_64x4096_bf16": _quant(64, 4096, "bf16"),
        # AlexNet's largest fully connected layer's weights, brought to 4 bits once at loading
        "quantize_4096x9216_f32": _quant(4096, 9216, "f32"),
        # one token through a square layer: a stream of 4-bit weights, where latency counts
        "fc_mx4_1x4096x4096_bf16": _fc(1, 4096, 4096, "bf16", False, False),
        # AlexNet's largest fully connected layer on a batch, in the library's own type
        "fc_mx4_64x9216x4096_f32": _fc(64, 9216, 4096, "f32", False, True),
        # the same layer on a long prompt, both operands in 4 bits
        "fc_mx4_2048x9216x4096_x4": _fc(2048, 9216, 4096, "bf16", True, False),
        # a long prompt through eight large experts: the largest products
        "grouped_4096x2of8_bf16": _grouped(4096, 8, 2, 4096, 4096, "bf16", False, True),
        # 16 sequences decode one token each: nearly every expert has a row or two, its weights in 4 bits
        "grouped_decode_16x4of64_mx4": _grouped(16, 64, 4, 2048, 4096, "bf16", True, True),
        # odd sizes throughout, in the library's own type
        "grouped_odd_77x3of7_f32": _grouped(77, 7, 3, 610, 1013, "f32", False, False),
        # the router of a long prompt
        "route_8192x8of64_bf16": _route(8192, 64, 8, "bf16", True),
        # the router of a small decode batch: the smallest call of all
        "route_16x4of128_f32": _route(16, 128, 4, "f32", False),
        # the experts' outputs of a long prompt back in token order
        "combine_4096x8x2048_bf16": _combine(4096, 8, 2048, "bf16"),
        # an odd width, a few tokens
        "combine_33x3x1013_f16": _combine(33, 3, 1013, "f16"),
    }
    return [{"name": name, **case} for name, case in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A layer's width: mostly a multiple of 64, as layers have, else any number."""
    w = _log_int(rng, lo, hi)
    return max(64, w // 64 * 64) if rng.random() < 0.6 else w


def draw(rng):
    most = max(2 * c["tokens"] * c["k"] * c["i"] * c["o"] for c in listed() if c["op"] == "grouped")
    u = rng.random()
    dtype = rng.choice(("f32", "bf16", "bf16", "f16"))
    if u < 0.15:
        return _quant(_log_int(rng, 1, 4096), _width(rng, 33, 9216), dtype)
    if u < 0.45:
        while True:
            case = _fc(_log_int(rng, 1, 4096), _width(rng, 64, 9216), _width(rng, 10, 8192), dtype,
                       rng.random() < 0.35, rng.random() < 0.5)
            if work(case)["flops"] <= most / (16 if dtype == "f32" else 1):
                return case
    if u < 0.75:
        while True:
            experts = _log_int(rng, 2, 128)
            case = _grouped(_log_int(rng, 1, 4096), experts, rng.randint(1, min(8, experts)), _width(rng, 64, 4096),
                            _width(rng, 64, 4096), dtype, rng.random() < 0.5, rng.random() < 0.5)
            small = experts * case["i"] * case["o"] <= 8 * 4096 * 4096
            if small and work(case)["flops"] <= most / (16 if dtype == "f32" else 1):
                return case
    if u < 0.90:
        experts = _log_int(rng, 2, 256)
        return _route(_log_int(rng, 1, 16384), experts, rng.randint(1, min(8, experts)), dtype, rng.random() < 0.5)
    return _combine(_log_int(rng, 1, 4096), rng.randint(1, 8), _width(rng, 64, 4096), dtype)


# ------------------------------------------------------------------ inputs
def _normal(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda")


def _activations(rows, cols, gen):
    """Normal values whose channels differ in size, some by a lot, as the activations inside large models do."""
    return _normal((rows, cols), gen) * torch.exp(0.5 * _normal((cols,), gen))


def _packed(rows, cols, fan, gen):
    """Weights in mx4, as a file holds them: bytes [rows][ceil(cols/32)*16], scales [rows][ceil(cols/32)]; the
    values behind the last column are zero."""
    blocks = -(-cols // 32)
    q = torch.randint(0, 256, (rows, blocks * 16), generator=gen, device="cuda", dtype=torch.uint8)
    at = 2 * torch.arange(blocks * 16, device="cuda")
    keep = 0x0F * (at < cols).to(torch.uint8) + 0xF0 * (at + 1 < cols).to(torch.uint8)
    # the 4-bit values have a mean square of 8: scales around 1 / sqrt(8 fan) keep the sums' size
    low = 127 - int(round(math.log2(8 * fan) / 2))
    scale = torch.randint(low - 2, low + 2, (rows, blocks), generator=gen, device="cuda", dtype=torch.uint8)
    return q & keep, scale


def _choices(tokens, experts, k, gen):
    """k different experts for every token, some more popular than others."""
    liked = 0.7 * _normal((experts,), gen)
    noise = -torch.log(-torch.log(torch.rand((tokens, experts), generator=gen, device="cuda").clamp(1e-7, 1 - 1e-6)))
    return (liked + noise).topk(k, dim=1).indices


def _by_expert(choice, experts):
    """(token of every slot, first slot of every expert, slot of every choice), slots ordered by expert, then token."""
    tokens, k = choice.shape
    order = torch.argsort(choice.reshape(-1), stable=True)
    slot = torch.empty_like(order)
    slot[order] = torch.arange(tokens * k, device=order.device)
    counts = (choice.reshape(-1, 1) == torch.arange(experts, device=choice.device)).sum(0)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    return (order // k).to(torch.int32), offsets.to(torch.int32), slot.reshape(tokens, k).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case}
    op, dtype = case["op"], _TYPES[case["dtype"]]
    if op == "quantize":
        s["x"] = _activations(case["rows"], case["cols"], gen).to(dtype)
    elif op == "fc_mx4":
        s["x"] = _activations(case["n"], case["i"], gen).to(dtype)
        s["w"], s["scale"] = _packed(case["o"], case["i"], case["i"], gen)
        s["b"] = 0.1 * _normal((case["o"],), gen)
    elif op == "grouped":
        e, i, o = case["experts"], case["i"], case["o"]
        s["x"] = _activations(case["tokens"], i, gen).to(dtype)
        if case["w4"]:
            q, scale = _packed(e * o, i, i, gen)
            s["w"], s["scale"] = q.reshape(e, o, -1), scale.reshape(e, o, -1)
        else:
            s["w"], s["scale"] = (_normal((e, o, i), gen) / math.sqrt(i)).to(dtype), None
        s["b"] = 0.1 * _normal((e, o), gen)
        s["rows"], s["offsets"], _ = _by_expert(_choices(case["tokens"], e, case["k"], gen), e)
        s["most"] = int((s["offsets"][1:] - s["offsets"][:-1]).max())
    elif op == "route":
        s["logits"] = (1.5 * _normal((case["tokens"], case["experts"]), gen)).to(dtype)
    else:
        t, k, d = case["tokens"], case["k"], case["d"]
        s["x"] = _activations(t * k, d, gen).to(dtype)
        s["weight"] = torch.softmax(_normal((t, k), gen), dim=1)
        _, _, s["slot"] = _by_expert(_choices(t, max(8, 2 * k), k, gen), max(8, 2 * k))
    return s


# ------------------------------------------------------------------ plain forms
def _blocks(x):
    """x [rows][cols] as [rows][blocks][32], zeros behind the last column."""
    rows, cols = x.shape
    return torch.nn.functional.pad(x, (0, -cols % 32)).reshape(rows, -1, 32)


def _two_to(e):
    """2^e in fp32 for whole e from -127 to 127, exactly (a library's power may be a rounding off)."""
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _through_mx4(x):
    """The mx4 values nearest to x (fp32), ties to the even mantissa."""
    b = _blocks(x)
    _, e = torch.frexp(b.abs().amax(-1, keepdim=True))
    e = (e - 3).clamp(min=-127)  # the largest value of a block gets the exponent of 4, the largest one's
    a = b.abs() * _two_to(-e)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp(max=6.0)
    return (torch.copysign(a, b) * _two_to(e)).reshape(x.shape[0], -1)[:, :x.shape[1]]


def _unpack(q, scale, cols):
    """The values of mx4 bytes and scales, in fp32."""
    code = torch.stack([q & 15, q >> 4], -1).flatten(-2).to(torch.int32)
    mag = code & 7
    small = 0.5 * mag
    large = (2 + (mag & 1)) * _two_to((mag >> 1) - 2)
    v = torch.where(mag < 2, small, large) * (1 - 2 * (code >> 3))
    v = v.reshape(*scale.shape, 32)
    return (v * _two_to(scale.to(torch.int32) - 127).unsqueeze(-1)).flatten(-2)[..., :cols]


def _plain_grouped(s):
    case = s["case"]
    e, offsets = case["experts"], s["offsets"].long()
    m = s["rows"].numel()
    slot = torch.arange(m, device=offsets.device)
    group = torch.searchsorted(offsets[1:], slot, right=True)
    at = slot - offsets[group]
    x = torch.zeros((e, s["most"], case["i"]), device=offsets.device)
    x[group, at] = s["x"].float()[s["rows"].long()]
    w = _unpack(s["w"], s["scale"], case["i"]) if case["w4"] else s["w"].float()
    y = torch.bmm(x, w.transpose(1, 2).contiguous())[group, at] + s["b"][group]
    return (torch.relu(y) if case["relu"] else y).to(s["x"].dtype)


def _plain_route(s):
    case = s["case"]
    logits = s["logits"].float()
    # a stable descending order gives ties to the lowest index
    chosen = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :case["k"]]
    p = torch.exp(logits - logits.amax(1, keepdim=True))
    weight = p.gather(1, chosen)
    weight = weight / (weight if case["renorm"] else p).sum(1, keepdim=True)
    rows, offsets, slot = _by_expert(chosen, case["experts"])
    return {"expert": chosen.to(torch.int32), "weight": weight, "rows": rows, "offsets": offsets, "slot": slot}


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "quantize":
        return _through_mx4(s["x"].float()).to(s["x"].dtype)
    if op == "fc_mx4":
        x = s["x"].float()
        x = _through_mx4(x) if case["x4"] else x
        y = x @ _unpack(s["w"], s["scale"], case["i"]).T + s["b"]
        return (torch.relu(y) if case["relu"] else y).to(s["x"].dtype)
    if op == "grouped":
        return _plain_grouped(s)
    if op == "route":
        return _plain_route(s)
    return (s["x"].float()[s["slot"].long()] * s["weight"].unsqueeze(-1)).sum(1).to(s["x"].dtype)


# ------------------------------------------------------------------ the library's calls
def _library(s):
    from paper_1511_07376_amd import cnn

    case = s["case"]
    op = case["op"]
    if op == "quantize":
        q, scale = cnn.cnn_mx4_quantize(s["x"])
        return cnn.cnn_mx4_dequantize(q, scale, case["cols"], dtype=s["x"].dtype)
    if op == "fc_mx4":
        if case["x4"]:
            xq, xs = cnn.cnn_mx4_quantize(s["x"])
            return cnn.cnn_fc_mx4_fwd(xq, s["w"], s["scale"], s["b"], case["relu"], x_scale=xs, y_dtype=s["x"].dtype)
        return cnn.cnn_fc_mx4_fwd(s["x"], s["w"], s["scale"], s["b"], case["relu"])
    if op == "grouped":
        return cnn.cnn_fc_grouped_fwd(s["x"], s["w"], s["offsets"], s["b"], case["relu"], rows=s["rows"],
                                      w_scale=s["scale"])
    if op == "route":
        expert, weight, rows, offsets, slot = cnn.cnn_route_fwd(s["logits"], case["k"], renormalize=case["renorm"])
        return {"expert": expert, "weight": weight, "rows": rows, "offsets": offsets, "slot": slot}
    return cnn.cnn_combine_fwd(s["x"], s["slot"], s["weight"])


def run(state):
    return _library(state) if own else _plain(state)


def work(case):
    op, sz = case["op"], _BYTES[case["dtype"]]
    if op == "quantize":
        n = case["rows"] * case["cols"]
        # read, write the 4-bit form, and back: read it, write the values
        return {"bytes": n * (2 * sz + 2 * _BYTES["mx4"]), "flops": 4 * n}
    if op == "fc_mx4":
        n, i, o = case["n"], case["i"], case["o"]
        return {"bytes": n * i * sz + o * i * _BYTES["mx4"] + 4 * o + n * o * sz, "flops": 2 * n * i * o}
    if op == "grouped":
        t, e, k, i, o = (case[key] for key in ("tokens", "experts", "k", "i", "o"))
        hit = e * (1 - (1 - k / e) ** t)  # experts that some token chooses
        w = _BYTES["mx4"] if case["w4"] else sz
        return {"bytes": t * i * sz + hit * o * (i * w + 4) + t * k * (o * sz + 4), "flops": 2 * t * k * i * o}
    if op == "route":
        t, e, k = case["tokens"], case["experts"], case["k"]
        return {"bytes": t * e * sz + 16 * t * k + 4 * e, "flops": t * e * (k + 3)}
    t, k, d = case["tokens"], case["k"], case["d"]
    return {"bytes": t * k * d * sz + t * d * sz + 8 * t * k, "flops": 2 * t * k * d}


# ------------------------------------------------------------------ 64 bits
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _quantized64(x):
    """mx4 values of x by search: the table entry nearest to |x| / scale, of two as near the one with an even code."""
    rows, cols = x.shape
    b = torch.nn.functional.pad(x.double(), (0, -cols % 32)).reshape(rows, -1, 32)
    top = b.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -149)
    # a double's bits without its mantissa are the power of two below it
    scale = ((top.view(torch.int64) >> 52) << 52).view(torch.float64).mul(0.25).clamp(min=2.0 ** -127)
    a = b.abs() / scale
    best, dist = torch.zeros_like(a), a.clone()
    for code, value in enumerate(_E2M1[1:], 1):
        d = (a - value).abs()
        take = (d < dist) | ((d == dist) & (code % 2 == 0))
        best, dist = torch.where(take, value, best), torch.where(take, d, dist)
    return (torch.sign(b) * best * scale).reshape(rows, -1)[:, :cols]


def _values64(q, scale, cols):
    table = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), dtype=torch.float64, device=q.device)
    v = torch.empty((*q.shape, 2), dtype=torch.float64, device=q.device)
    v[..., 0] = table[(q % 16).long()]
    v[..., 1] = table[torch.div(q, 16, rounding_mode="floor").long()]
    v = v.reshape(*q.shape[:-1], -1) * ((scale.long() + 896) << 52).view(torch.float64).repeat_interleave(32, dim=-1)
    return v[..., :cols]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        return _quantized64(s["x"])
    if op == "fc_mx4":
        x = _quantized64(s["x"]) if case["x4"] else s["x"].double()
        y = torch.addmm(s["b"].double(), x, _values64(s["w"], s["scale"], case["i"]).T)
        return y.clamp(min=0) if case["relu"] else y
    if op == "grouped":
        bounds = s["offsets"].tolist()
        y = torch.empty((bounds[-1], case["o"]), dtype=torch.float64, device="cuda")
        for g in range(case["experts"]):
            lo, hi = bounds[g], bounds[g + 1]
            w = _values64(s["w"][g], s["scale"][g], case["i"]) if case["w4"] else s["w"][g].double()
            y[lo:hi] = s["x"][s["rows"][lo:hi].long()].double() @ w.T + s["b"][g].double()
        return y.clamp(min=0) if case["relu"] else y
    if op == "route":
        p = torch.softmax(s["logits"].double(), dim=1)
        # as p falls with the logit, its k largest values are those of the choices, in their order
        weight = p.sort(dim=1, descending=True).values[:, :case["k"]]
        weight = weight / weight.sum(1, keepdim=True) if case["renorm"] else weight
        return {"expert": None, "weight": weight, "rows": None, "offsets": None, "slot": None}
    y = torch.zeros((case["tokens"], case["d"]), dtype=torch.float64, device="cuda")
    for j in range(case["k"]):
        y += s["weight"][:, j:j + 1].double() * s["x"][s["slot"][:, j].long()].double()
    return y
