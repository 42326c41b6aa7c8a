"""The optimizer step behind the exchange of compressed gradients, as timed cases.

Three operators over the layers of one flat buffer:
  norms   sum of the squared gradients of every layer and of all of them
  adamw   AdamW with decoupled weight decay, fp32 moments; with `clip` the norms first, and the gradients scaled by them
  coded   the same with moments in 8 bits (blocks of 128 elements with an exponent each), and the moments' values

Coded moments.  A block of 128 elements, counted from its layer's start, has two bytes x: the biased fp32 exponent of its
largest |m| (of its largest v), one more where the mantissa exceeds 31/16.  A code holds a magnitude below 2 * 2^(x-127)
with 4 mantissa bits: exponents 0 .. -6 below the block's (m, behind a sign bit) or 0 .. -14 (v), and steps of the lowest
exponent below that.  Rounding is to the nearest, ties to even codes, or stochastic: up where the part cut off, plus
u = (r + 1/2) / 2^16, reaches a step; r is the lower (m) or upper (v) half of word i % 4 of Philox4x32-10 with the seed as key
and the counter (i / 4, step, layer, 1), i the element's index in its layer.  A v above zero keeps at least the lowest step.
The parameters are updated from the moments before they are rounded.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 128
BETA1, BETA2, EPS = 0.9, 0.999, 1e-8


def listed():
    return [
        # clipping's norm for a toy model: launches and the host's part are all of it
        {"name": "norms_tiny", "op": "norms", "model": "tiny", "grads": "f32"},
        # odd channel counts: nearly every layer starts off alignment; 16-bit gradients
        {"name": "norms_ragged_convnet_bf16", "op": "norms", "model": "convnet", "layers": 13, "width": 211,
         "classes": 101, "grads": "bf16"},
        # the largest gradient buffer
        {"name": "norms_gpt2_medium", "op": "norms", "model": "gpt2", "layers": 24, "width": 1024, "vocab": 50257,
         "grads": "f32"},
        # the smallest step
        {"name": "adamw_tiny", "op": "adamw", "model": "tiny", "grads": "f32", "copy": "none", "clip": False,
         "skip": 0},
        # thousands of short tensors (adapters, biases and norms of a deep model)
        {"name": "adamw_many_small", "op": "adamw", "model": "many", "layers": 4000, "width": 700, "grads": "f32",
         "copy": "none", "clip": True, "skip": 3},
        # an image classifier
        {"name": "adamw_resnet50", "op": "adamw", "model": "resnet50", "classes": 1000, "grads": "f32", "copy": "none",
         "clip": False, "skip": 0},
        # a language model in mixed precision: gradients and the forward pass's weights in bf16
        {"name": "adamw_transformer_lm_bf16", "op": "adamw", "model": "transformer_lm", "layers": 16, "width": 512,
         "vocab": 32768, "grads": "bf16", "copy": "bf16", "clip": True, "skip": 0},
        # the largest with fp32 moments: the receiver's fp32 gradients, clipped
        {"name": "adamw_gpt2_medium", "op": "adamw", "model": "gpt2", "layers": 24, "width": 1024, "vocab": 50257,
         "grads": "f32", "copy": "none", "clip": True, "skip": 0},
        # 8-bit moments, smallest
        {"name": "coded_tiny", "op": "coded", "model": "tiny", "grads": "f32", "copy": "none", "clip": False, "skip": 0,
         "stochastic": True},
        # 8-bit moments of ragged layers behind gaps: blocks that end early, nothing aligned
        {"name": "coded_ragged_convnet", "op": "coded", "model": "convnet", "layers": 13, "width": 211, "classes": 101,
         "grads": "f32", "copy": "f16", "clip": True, "skip": 5, "stochastic": True},
        # 8-bit moments, rounded to nearest
        {"name": "coded_resnet50_nearest", "op": "coded", "model": "resnet50", "classes": 1000, "grads": "f32",
         "copy": "none", "clip": False, "skip": 0, "stochastic": False},
        # the largest in the least memory: bf16 gradients and weights, 8-bit moments, stochastic rounding
        {"name": "coded_gpt2_medium_bf16", "op": "coded", "model": "gpt2", "layers": 24, "width": 1024, "vocab": 50257,
         "grads": "bf16", "copy": "bf16", "clip": True, "skip": 0, "stochastic": True},
    ]


def draw(rng):
    n = math.exp(rng.uniform(math.log(200), math.log(250_000_000)))
    case = {"op": rng.choice(["norms", "adamw", "adamw", "coded", "coded"]),
            "model": rng.choice(["convnet", "gpt2", "transformer_lm", "many"]), "grads": rng.choice(["f32", "f32", "bf16"])}
    if case["model"] == "many":
        case["layers"] = max(1, min(int(n / rng.randint(40, 1500)), rng.randint(1, 6000)))
        case["width"] = max(1, int(n / case["layers"]))
    elif case["model"] == "convnet":
        case["layers"] = rng.randint(2, 20)
        case.update(width=max(3, int(math.sqrt(n / (9.0 * case["layers"])))), classes=rng.randint(2, 1000))
    else:
        case["layers"] = rng.randint(1, 24)
        width = math.sqrt(0.7 * n / (12.0 * case["layers"]))
        case["width"] = max(2, int(width)) if rng.random() < 0.5 else max(16, int(width) // 16 * 16)
        case["vocab"] = max(7, int(0.3 * n / case["width"]))
    if case["op"] != "norms":
        case.update(copy=rng.choice(["none", "bf16", "f16"]), clip=rng.random() < 0.6, skip=rng.choice([0, 0, 1, 4, 32]))
    if case["op"] == "coded":
        case["stochastic"] = rng.random() < 0.6
    return case


# ------------------------------------------------------------------------------ what a case stands for
def _bottlenecks(planes, inp, blocks):
    first = [(planes, inp, 1, 1), (planes,), (planes,), (planes, planes, 3, 3), (planes,), (planes,),
             (4 * planes, planes, 1, 1), (4 * planes,), (4 * planes,)]
    rest = [(planes, 4 * planes, 1, 1)] + first[1:]
    return first + [(4 * planes, inp, 1, 1), (4 * planes,), (4 * planes,)] + rest * (blocks - 1)


def _shapes(case):
    m = case["model"]
    if m == "tiny":
        return [(16, 3, 3, 3), (32, 16, 3, 3), (64, 32, 3, 3), (10, 256)]
    if m == "resnet50":
        return ([(64, 3, 7, 7), (64,), (64,)] + _bottlenecks(64, 64, 3) + _bottlenecks(128, 256, 4) +
                _bottlenecks(256, 512, 6) + _bottlenecks(512, 1024, 3) + [(case["classes"], 2048), (case["classes"],)])
    w, n = case["width"], case["layers"]
    if m == "convnet":
        return [(w, 3, 3, 3), (w,)] + [(w, w, 3, 3), (w,)] * (n - 1) + [(case["classes"], w), (case["classes"],)]
    if m == "many":                                           # lengths around the width, most of them odd
        return [(1 + (2 * w - 1) * ((7919 * k + 500) % 1009) // 1008,) for k in range(n)]
    if m == "transformer_lm":
        block = [(w,)] * 2 + [(w, w), (w,)] * 4 + [(w,)] * 2 + [(4 * w, w), (4 * w,), (w, 4 * w), (w,)]
        return [(case["vocab"], w)] + block * n + [(w,)] * 2
    block = [(w,)] * 2 + [(w, 3 * w), (3 * w,), (w, w), (w,)] + [(w,)] * 2 + [(w, 4 * w), (4 * w,), (4 * w, w), (w,)]
    return [(case["vocab"], w), (1024, w)] + block * n + [(w,)] * 2


def _table(case):
    """Offsets and sizes of the layers, `skip` unused elements in front of each, and which are matrices."""
    shapes = _shapes(case)
    sizes = np.array([int(np.prod(s)) for s in shapes], np.int64)
    ends = np.cumsum(sizes + case.get("skip", 0))
    return ends - sizes, sizes, np.array([len(s) >= 2 for s in shapes])


_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def prepare(case, seed):
    op, dev = case["op"], torch.device("cuda")
    offsets, sizes, matrix = _table(case)
    total = int(offsets[-1] + sizes[-1]) + 1                  # an element behind the last layer, no layer's own
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    # decay for matrices only; the embedding (or first layer) learns at half the rate
    lr_scale = np.where(np.arange(len(sizes)) == 0, 0.5, 1.0).astype(np.float32)
    decay_scale = np.where(matrix, 1.0, 0.0).astype(np.float32)
    s = {"op": op, "lr": 10.0 ** rng.uniform(-4.0, -2.5), "decay": 0.1, "max_norm": 1.0, "seed": seed,
         "scale": 1.0 / rng.uniform(3.0, 5.0),                # a mean over workers with unlike numbers of tokens
         "clip": case.get("clip", False), "stochastic": case.get("stochastic", False)}
    # the blocks of the layers: their elements' places in the buffer (dead places: the element behind the last layer)
    per = (sizes + BLOCK - 1) // BLOCK
    firsts = np.cumsum(per) - per
    layer = torch.from_numpy(np.repeat(np.arange(len(sizes)), per)).to(dev)
    at_layer = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)[layer]  # noqa: E731
    index = ((torch.arange(len(layer), device=dev) - at_layer(firsts)) * BLOCK)[:, None] + torch.arange(BLOCK, device=dev)
    live = index < at_layer(sizes)[:, None]
    at = torch.where(live, index + at_layer(offsets)[:, None], total - 1)
    s.update(layer=layer, at=at, live=live, first=at_layer(firsts),
             ends=torch.from_numpy(np.cumsum(per)).to(dev), lr_scale=at_layer(lr_scale), decay_scale=at_layer(decay_scale))
    del index
    # gradients of every layer at a scale of its own
    spread = at_layer((10.0 ** rng.uniform(-4.5, -2.0, len(sizes))).astype(np.float32))[:, None]

    def made(values, dtype=torch.float32):
        out = torch.zeros(total, dtype=dtype, device=dev)
        out[at] = torch.where(live, values, 0).to(dtype)
        return out

    normal = lambda: torch.randn(at.shape, generator=gen, device=dev)  # noqa: E731
    s["g"] = made(normal() * spread, _TYPES[case["grads"]])
    if op != "norms":
        s["p"] = made(normal() * 0.02)
        s["step"] = torch.tensor([int(rng.integers(0, 2000))], device=dev)
        m = normal() * spread * (0.25 * 0.2)
        v = (normal().square() + 0.5) * (spread * 0.25).square()
        if op == "adamw":
            s["m"], s["v"] = made(m), made(v)
        else:
            s["m"], s["v"], s["x"] = _encoded(torch.where(live, m, 0), torch.where(live, v, 0), at, total)
        if case["copy"] != "none":
            s["copy"] = torch.zeros(total, dtype=_TYPES[case["copy"]], device=dev)
    if op == "coded":
        s["m_values"] = torch.zeros(total, dtype=torch.bfloat16, device=dev)
        s["v_values"] = torch.zeros(total, dtype=torch.bfloat16, device=dev)
    s["sumsq"] = torch.zeros(len(sizes) + 1, dtype=torch.float64, device=dev)
    if own:
        from paper_2210_17357_amd import binding as B
        zero = np.zeros(len(sizes), np.int32)
        s["plan"] = B.Optim(B.layer_table(offsets, sizes, zero, zero), lr_scale, decay_scale)
        s["settings"] = B.adamw(lr=s["lr"], beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=s["decay"],
                                grad_scale=s["scale"], max_norm=s["max_norm"] if s["clip"] else 0.0,
                                stochastic=s["stochastic"], seed=seed)
    return s


# ------------------------------------------------------------------------------ the plain form
def _block_exponent(a):
    """The exponent byte of blocks with these magnitudes."""
    bits = a.amax(1).view(torch.int32)
    return (bits + 0x7FFFF) >> 23


def _power(e):
    return torch.pow(2.0, e.double())


def _rounded(a, x, octaves, u=None):
    """Magnitudes as whole steps of their octave, and those steps: a = q * step."""
    ratio = a.double() / _power(x - 127)[:, None]
    e = torch.floor(torch.log2(ratio.clamp(min=2.0 ** (1 - octaves))))
    e = torch.where(torch.pow(2.0, e) > ratio, e - 1, e).clamp(min=1 - octaves)
    e = torch.where(torch.pow(2.0, e + 1) <= ratio, e + 1, e)
    step = torch.pow(2.0, e - 4)
    q = ratio / step
    return (torch.round(q) if u is None else torch.floor(q + u)), step


def _code(q, step, octaves):
    """The byte (or 7 bits) of a rounded magnitude: 16 codes an octave above the lowest."""
    e = torch.log2(step).round() + 4
    return torch.where(q < 16, q, q + 16 * (e + octaves - 1))


def _encoded(m, v, at, total):
    x = torch.stack((_block_exponent(m.abs()), _block_exponent(v)), 1)
    cm = _code(*_rounded(m.abs(), x[:, 0], 7), 7) + 128 * (m < 0)
    cv = _code(*_rounded(v, x[:, 1], 15), 15)
    cv = torch.where(v > 0, cv.clamp(min=1), cv)
    out = [torch.zeros(total, dtype=torch.uint8, device=m.device) for _ in range(2)]
    out[0][at], out[1][at] = cm.to(torch.uint8), cv.to(torch.uint8)
    return out[0], out[1], x.to(torch.uint8)


def _decoded(code, x):
    """Values of codes without sign: exponent field and four mantissa bits, the lowest field without the leading one."""
    code = code.to(torch.int32)
    field, f = code >> 4, code & 15
    whole = torch.where(field > 0, (16 + f).double() * _power(field - 1), f.double())
    return whole, x


def _random_words(s, t):
    """Philox4x32-10's word of every element of the blocks."""
    mask = 0xFFFFFFFF

    def times(k, a):                                          # the two halves of a product of 32-bit numbers
        low, high = (k & 0xFFFF) * a, (k >> 16) * a
        mid = (low >> 16) + (high & mask)
        return (high >> 32 << 16) + (mid >> 16) & mask, ((mid & 0xFFFF) << 16) | (low & 0xFFFF)

    b = torch.arange(len(s["layer"]), device=s["layer"].device) - s["first"]
    c0 = b[:, None] * (BLOCK // 4) + torch.arange(BLOCK // 4, device=b.device)
    c1, c2 = torch.zeros_like(c0) + (t & mask), torch.zeros_like(c0) + s["layer"][:, None]
    c3 = torch.zeros_like(c0) + 1 + (t >> 32)
    k0, k1 = s["seed"] & mask, s["seed"] >> 32 & mask
    for _ in range(10):
        (h0, l0), (h1, l1) = times(0xD2511F53, c0), times(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = k0 + 0x9E3779B9 & mask, k1 + 0xBB67AE85 & mask
    return torch.stack((c0, c1, c2, c3), 2).view(-1, BLOCK)


def _put(buffer, at, live, values):
    buffer[at] = torch.where(live, values.to(buffer.dtype), buffer[-1])


def _norms(s):
    squares = torch.where(s["live"], s["g"][s["at"]].double().square(), 0).sum(1)
    upto = torch.cat((squares.new_zeros(1), squares.cumsum(0)))[torch.cat((s["ends"].new_zeros(1), s["ends"]))]
    s["sumsq"][:-1] = upto.diff()
    s["sumsq"][-1] = squares.sum()


def _step(s):
    at, live = s["at"], s["live"]
    scale, ok = torch.tensor(s["scale"], dtype=torch.float64, device=at.device), True
    if s["clip"]:
        ok = torch.isfinite(s["sumsq"][-1])
        scale = scale * (s["max_norm"] / (s["sumsq"][-1].sqrt() * s["scale"] + 1e-6)).clamp(max=1.0)
    t = s["step"] + 1
    g = s["g"][at].float() * scale.float()
    p = s["p"][at]
    if s["op"] == "adamw":
        m_old, v_old = s["m"][at], s["v"][at]
    else:
        c, x = s["m"][at], s["x"].to(torch.int32)
        a, e = _decoded(c & 127, x[:, 0])
        m_old = (a * _power(e - 127 - 10)[:, None] * torch.where(c > 127, -1.0, 1.0)).float()
        a, e = _decoded(s["v"][at], x[:, 1])
        v_old = (a * _power(e - 127 - 18)[:, None]).float()
    m = m_old * BETA1 + g * (1.0 - BETA1)
    v = v_old * BETA2 + g * g * (1.0 - BETA2)
    c1, c2 = 1.0 - torch.pow(BETA1, t.double()), 1.0 - torch.pow(BETA2, t.double())
    rate = s["lr"] * s["lr_scale"][:, None].double()
    shrink = (rate * s["decay"] * s["decay_scale"][:, None].double()).float()
    new = p - (p * shrink + (rate / c1).float() * m / (v.sqrt() * (1.0 / c2.sqrt()).float() + EPS))
    live = live & ok
    _put(s["p"], at, live, new)
    if "copy" in s:
        _put(s["copy"], at, live, new)
    if s["op"] == "adamw":
        _put(s["m"], at, live, m)
        _put(s["v"], at, live, v)
    else:
        m, v = torch.where(live, m, 0), torch.where(live, v, 0)
        xm, xv, um, uv = _block_exponent(m.abs()), _block_exponent(v), None, None
        if s["stochastic"]:
            r = _random_words(s, t)
            um, uv = ((r & 0xFFFF) + 0.5).double() / 65536, ((r >> 16) + 0.5).double() / 65536
        qm, step_m = _rounded(m.abs(), xm, 7, um)
        qv, step_v = _rounded(v, xv, 15, uv)
        qv = torch.where(v > 0, qv.clamp(min=1), qv)
        _put(s["m"], at, live, _code(qm, step_m, 7) + 128 * (m < 0))
        _put(s["v"], at, live, _code(qv, step_v, 15))
        s["x"].copy_(torch.where(torch.as_tensor(ok, device=at.device), torch.stack((xm, xv), 1), s["x"]))
        _put(s["m_values"], at, live, (qm * step_m * _power(xm - 127)[:, None] * torch.where(m < 0, -1.0, 1.0)).float())
        _put(s["v_values"], at, live, (qv * step_v * _power(xv - 127)[:, None]).float())
    s["step"] += torch.as_tensor(ok, device=at.device).long()


def run(s):
    op = s["op"]
    if own:
        plan = s["plan"]
        if op == "norms" or s["clip"]:
            plan.norms(s["g"], s["sumsq"])
        clip = s["sumsq"] if s["clip"] else None
        if op == "adamw":
            plan.adamw(s["settings"], s["g"], s["p"], s["m"], s["v"], s["step"], d_copy=s.get("copy"), d_sumsq=clip)
        elif op == "coded":
            plan.adamw_coded(s["settings"], s["g"], s["p"], s["m"], s["v"], s["x"], s["step"], d_copy=s.get("copy"),
                             d_sumsq=clip)
            plan.decode(s["m"], s["v"], s["x"], s["m_values"], s["v_values"])
    else:
        if op == "norms" or s["clip"]:
            _norms(s)
        if op != "norms":
            _step(s)
    if op == "norms":
        return s["sumsq"]
    out = [s["p"], s["step"], s["sumsq"]]
    out += [s["m"], s["v"]] if op == "adamw" else [s["m_values"], s["v_values"]]
    return out + ([s["copy"]] if "copy" in s else [])


def work(case):
    """Gradients read once, parameters and moments read and written, copies, norms and moments' values written."""
    _, sizes, _ = _table(case)
    n, blocks = float(sizes.sum()), float(((sizes + BLOCK - 1) // BLOCK).sum())
    grads = {"f32": 4.0, "bf16": 2.0}[case["grads"]]
    if case["op"] == "norms":
        return {"bytes": grads * n + 8.0 * (len(sizes) + 1), "flops": 2.0 * n}
    b = grads + 8.0 + (2.0 if case["copy"] != "none" else 0.0)
    if case["op"] == "adamw":
        return {"bytes": (b + 16.0) * n, "flops": 16.0 * n}
    return {"bytes": (b + 4.0 + 4.0) * n + 4.0 * blocks, "flops": 16.0 * n}


# ------------------------------------------------------------------------------ the definition in 64 bits
def _exact_words(seed, step, layer, n, device):
    """The random words of a layer's elements; products of 32-bit numbers split at 12 bits of one factor."""
    low32 = (1 << 32) - 1
    i = torch.arange((n + 3) // 4, device=device)
    c = [i, torch.full_like(i, step & low32), torch.full_like(i, layer), torch.full_like(i, 1 + (step >> 32))]
    key = [seed & low32, seed >> 32 & low32]
    for _ in range(10):
        halves = []
        for k, a in ((0xD2511F53, c[0]), (0xCD9E8D57, c[2])):
            top, mid, low = (k >> 24) * a, (k >> 12 & 0xFFF) * a, (k & 0xFFF) * a
            s1 = mid + (low >> 12)                            # the product without its lowest 12 bits, top part apart
            s2 = top + (s1 >> 12)
            halves.append((s2 >> 8, ((s2 & 0xFF) << 24) | ((s1 & 0xFFF) << 12) | (low & 0xFFF)))
        (h0, l0), (h1, l1) = halves
        c = [h1 ^ c[1] ^ key[0], l1, h0 ^ c[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) & low32, (key[1] + 0xBB67AE85) & low32]
    return torch.stack(c, 1).reshape(-1)[:n]


def _exact_stored(a, octaves, u):
    """What 8 bits keep of one layer's magnitudes (fp64, a multiple of 128 of them)."""
    blocks = a.view(-1, BLOCK)
    mant, exp = torch.frexp(blocks.amax(1))                   # amax = mant * 2^exp, mant in [1/2, 1)
    top = exp.double() - 1 + (mant * 2 > 31 / 16)
    _, e = torch.frexp(blocks)
    e = torch.maximum(e.double() - 1, top[:, None] - (octaves - 1))
    q = blocks * torch.pow(2.0, 4 - e)
    q = torch.round(q) if u is None else torch.floor(q + u.view(-1, BLOCK))
    return (q * torch.pow(2.0, e - 4)).view(-1), torch.pow(2.0, top - (octaves - 1) - 4)[:, None].expand_as(blocks).reshape(-1)


def exact(case, seed):
    s = prepare(case, seed)
    offsets, sizes, matrix = _table(case)
    op, n_layers = case["op"], len(sizes)
    if n_layers > 1000 and op == "coded":
        return None                                           # a layer at a time takes too long
    g_all = s["g"]
    sums = [g_all[o:o + n].double().square().sum() for o, n in zip(offsets.tolist(), sizes.tolist())]
    sumsq = torch.stack(sums + [torch.stack(sums).sum()])
    if op == "norms":
        return sumsq
    c = s["scale"]
    if s["clip"]:
        c = c * min(1.0, s["max_norm"] / (math.sqrt(float(sumsq[-1])) * s["scale"] + 1e-6))
    t = int(s["step"]) + 1
    outs = [torch.zeros(len(g_all), dtype=torch.float64, device=g_all.device) for _ in range(3)]
    first = 0
    for k, (o, n) in enumerate(zip(offsets.tolist(), sizes.tolist())):
        cut = slice(o, o + n)
        g, p = g_all[cut].double() * c, s["p"][cut].double()
        blocks = -(-n // BLOCK)
        if op == "adamw":
            m, v = s["m"][cut].double(), s["v"][cut].double()
        else:
            x = s["x"][first:first + blocks].double().repeat_interleave(BLOCK, 0)[:n]
            cm, cv = s["m"][cut].long(), s["v"][cut].long()
            em, ev = (cm & 127) // 16, cv // 16
            m = torch.where(em == 0, cm % 16 / 8.0, 1 + cm % 16 / 16.0) * torch.pow(2.0, em + x[:, 0] - 134)
            m = torch.where(cm >= 128, -m, m)
            v = torch.where(ev == 0, cv % 16 / 8.0, 1 + cv % 16 / 16.0) * torch.pow(2.0, ev + x[:, 1] - 142)
        m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g.square()
        rate = s["lr"] * (0.5 if k == 0 else 1.0)
        update = (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + EPS)
        outs[0][cut] = p - rate * (update + (s["decay"] * p if matrix[k] else 0.0))
        if op == "coded":
            um = uv = None
            pad = blocks * BLOCK - n
            if s["stochastic"]:
                r = torch.nn.functional.pad(_exact_words(s["seed"], t, k, n, g.device), (0, pad))
                um, uv = (2 * (r % 65536) + 1).double() / 131072, (2 * (r // 65536) + 1).double() / 131072
            km, _ = _exact_stored(torch.nn.functional.pad(m.abs(), (0, pad)), 7, um)
            kv, least = _exact_stored(torch.nn.functional.pad(v, (0, pad)), 15, uv)
            m, v = torch.sign(m) * km[:n], torch.where(v > 0, torch.maximum(kv, least)[:n], kv[:n])
        outs[1][cut], outs[2][cut] = m, v
        first += blocks
    got = [outs[0], None, sumsq if s["clip"] else s["sumsq"], outs[1], outs[2]]
    return got + ([outs[0]] if "copy" in s else [])
