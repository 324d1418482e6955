"""Cases and plain forms of 4-bit layers and of gradients clipped by their norm (include/silenzio_clear.h).

A case is a dict of plain values with a "kind":
  linear   x [tokens][inner] floating times 4-bit weights [outer][inner] that the program keeps, a scale for every `group` of a row's entries
  round    w [outer][inner] to 4 bits, and back to the values that these stand for
  train    one step of a layer with 4-bit weights: w quantised, y, and with dy the gradients of x and of w's values
  clip     the gradients of an MLP of these widths, a bias for each layer, `layers` of them: their common norm, and all of them times what brings it
           down to 1 ("over": they are above it), in the places that they have in a bucket of each type
"dtype" is the type of the floating inputs and outputs (clip: "mixed" has 32-bit biases next to bf16 matrices); "slack" is how many elements the
rows of the first input lie further apart than they are long.

4-bit rows as the operators take them: blocks of 128 entries, 16 words of 32 bits each.  Word 4 j + s of a block has the entries 32 s + 8 j to
32 s + 8 j + 7, the first four in the low halves of its bytes and the others in the high halves, each a sign (the highest bit) and a magnitude.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "mixed": torch.bfloat16}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-6


def _layer(name, kind, tokens, inner, outer, dtype="bf16", group=128, slack=0):
    return dict(name=name, kind=kind, tokens=tokens, inner=inner, outer=outer, dtype=dtype, group=group, slack=slack)


def _clip(name, widths, layers, dtype, over):
    return dict(name=name, kind="clip", widths=widths, layers=layers, dtype=dtype, over=over)


def listed():
    return [
        # one token through a layer whose weights stay in 4 bits: a step of serving
        _layer("linear_1x4096x8192", "linear", 1, 4096, 8192),
        # the first layer of the library's MLP (784 -> 128) on a mini-batch of 32 images; its last group of a row is half a group
        _layer("linear_32x784x128", "linear", 32, 784, 128, "f32", 32),
        # a few sequences at once, no size a multiple of anything
        _layer("linear_7x1555x1001", "linear", 7, 1555, 1001, "f16", 64, 5),
        # a step of serving 64 sequences
        _layer("linear_64x4096x16384", "linear", 64, 4096, 16384),
        # a long prompt through a wide layer
        _layer("linear_8192x8192x8192", "linear", 8192, 8192, 8192, "f16"),
        # the library's 784 -> 128 layer, as a step of training rounds it
        _layer("round_128x784", "round", 0, 784, 128, "f32", 32),
        # a wide layer before it is served
        _layer("round_8192x8192", "round", 0, 8192, 8192),
        # a training step with a ragged batch
        _layer("train_777x1001x1555", "train", 777, 1001, 1555, "f16", 64, 3),
        # a training step of a square layer
        _layer("train_4096x4096x4096", "train", 4096, 4096, 4096),
        # the gradients of the library's MLP: six small tensors
        _clip("clip_784x128x64x10", "784x128x64x10", 1, "f32", True),
        # many small tensors, late in training: below the limit
        _clip("clip_250x96x33x96", "96x33x96", 250, "f16", False),
        # a large model's step
        _clip("clip_8x4096x8192x4096", "4096x8192x4096", 8, "mixed", True),
    ]


def _log(rng, low, high):
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    kind = rng.choice(("linear", "linear", "linear", "round", "train", "clip", "clip"))
    while True:
        if kind == "clip":
            widths = "x".join(str(_log(rng, 8, 8192)) for _ in range(rng.choice((2, 3, 4))))
            c = _clip("", widths, _log(rng, 1, 250), rng.choice(("bf16", "f16", "f32", "mixed")), rng.choice((True, False)))
            fits = sum(math.prod(s) for s, _ in _tensors(c)) <= 2 ** 28
        else:
            c = _layer("", kind, _log(rng, 1, 8192), _log(rng, 32, 8192), _log(rng, 32, 8192), rng.choice(("bf16", "bf16", "f16", "f32")),
                       rng.choice((32, 64, 128, 128)), rng.choice((0, 0, 1, 8)))
            fits = work(c)["flops"] <= (4.2e11 if kind == "train" or c["dtype"] == "f32" else 1.1e12)
            if kind == "round":
                c["tokens"] = 0
        if fits:
            del c["name"]
            return c


def _tensors(case):
    """(shape, whether it is a bias) of each gradient of a clip case."""
    widths = [int(w) for w in case["widths"].split("x")]
    return [t for _ in range(case["layers"]) for k, n in zip(widths, widths[1:]) for t in (((n, k), False), ((n,), True))]


def _buckets(tensors):
    """How many elements the bucket of each type has: the tensors begin at multiples of 64."""
    sizes = {}
    for g in tensors:
        sizes[g.dtype] = sizes.get(g.dtype, 0) + (g.numel() + 63) // 64 * 64
    return sizes


def _places(tensors, buckets):
    views, at = [], {b.dtype: 0 for b in buckets}
    of = {b.dtype: b for b in buckets}
    for g in tensors:
        views.append(of[g.dtype][at[g.dtype]:at[g.dtype] + g.numel()].view(g.shape))
        at[g.dtype] += (g.numel() + 63) // 64 * 64
    return views


def _rows(gen, rows, cols, dtype, slack, std):
    """Values of a row-major matrix whose rows lie `slack` elements further apart than they are long."""
    return (torch.randn((rows, cols + slack), device="cuda", generator=gen) * std).to(TYPES[dtype])[:, :cols]


def _pack(q):
    """Whole numbers from -7 to 7 [rows][cols] to 4-bit rows."""
    rows, cols = q.shape
    blocks = (cols + 127) // 128
    code = torch.zeros((rows, blocks * 128), dtype=torch.uint8, device=q.device)
    code[:, :cols] = (q.abs() + 8 * (q < 0)).to(torch.uint8)
    code = code.view(rows, blocks, 4, 4, 2, 4).transpose(2, 3)             # [rows][block][j][s][half][byte]
    return (code[..., 0, :] + 16 * code[..., 1, :]).reshape(rows, blocks * 64)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind, s = case["kind"], {"kind": case["kind"], "dtype": TYPES[case["dtype"]]}
    if kind == "clip":
        tensors = _tensors(case)
        # noise of a common size, as after an initialisation that keeps variances
        std = (3.3 if case["over"] else 0.3) / math.sqrt(sum(math.prod(shape) for shape, _ in tensors))
        kinds = [torch.float32 if bias and case["dtype"] == "mixed" else s["dtype"] for _, bias in tensors]
        s["g"] = [(torch.randn(shape, device="cuda", generator=gen) * std).to(t) for (shape, _), t in zip(tensors, kinds)]
        s["buckets"] = [torch.zeros(n, dtype=t, device="cuda") for t, n in _buckets(s["g"]).items()]
        s["out"] = _places(s["g"], s["buckets"])
        return s
    M, K, N, dtype, slack = (case[k] for k in ("tokens", "inner", "outer", "dtype", "slack"))
    s["group"] = case["group"]
    if kind in ("linear", "train"):
        # activations after a norm: unit variance, a few channels larger
        s["x"] = _rows(gen, M, K, dtype, slack, 1.0)
        s["x"][:, ::61] *= 4
    if kind == "linear":
        s["q"] = _pack((torch.randn((N, K), device="cuda", generator=gen) * 2.6).round().clamp(-7, 7))
        s["scale"] = (torch.rand((N, (K + case["group"] - 1) // case["group"]), device="cuda", generator=gen) + 0.5) / (2.6 * math.sqrt(K))
    else:
        s["w"] = _rows(gen, N, K, dtype, slack if kind == "round" else 0, 1 / math.sqrt(K))
    if kind == "train":
        s["dy"] = _rows(gen, M, N, dtype, 0, 1 / math.sqrt(N))
    return s


def _unpack(q, cols):
    rows, blocks = q.shape[0], q.shape[1] // 64
    b = q.view(rows, blocks, 4, 4, 4)
    code = torch.stack((b & 15, b >> 4), dim=4).transpose(2, 3).reshape(rows, blocks * 128)[:, :cols]
    return torch.where(code >= 8, -1.0, 1.0) * (code & 7).float()


def _spread(scale, group, cols):
    return scale.repeat_interleave(group, dim=1)[:, :cols]


def _quantised(w, group):
    """Rows to whole numbers from -7 to 7 and a scale for every `group` entries.  In 64 bits: quotients next to a half decide between two numbers."""
    rows, cols = w.shape
    full = torch.zeros((rows, (cols + group - 1) // group * group), dtype=torch.float64, device=w.device)
    full[:, :cols] = w.double()
    x = full.view(rows, -1, group)
    top = x.abs().amax(2, keepdim=True)
    q = torch.round(7.0 * x / torch.where(top > 0, top, torch.ones_like(top))).view(rows, -1)[:, :cols]
    return q.float(), (top[:, :, 0].float() / 7.0)


def _plain(s):
    kind, out = s["kind"], s["dtype"]
    if kind == "clip":
        total = torch.zeros((), dtype=torch.float64, device="cuda")
        for g in s["g"]:
            f = g.float()
            total = total + (f * f).sum().double()
        norm = torch.sqrt(total).float()
        by = torch.clamp(1.0 / (norm + EPS), max=1.0)
        for g, o in zip(s["g"], s["out"]):
            o.copy_(g.float() * by)
        return [norm] + s["buckets"]
    group = s["group"]
    if kind == "linear":
        cols = s["x"].shape[1]
        w = _unpack(s["q"], cols) * _spread(s["scale"], group, cols)
        return {"y": (s["x"].float() @ w.t()).to(out)}
    q, scale = _quantised(s["w"], group)
    w = q * _spread(scale, group, q.shape[1])
    if kind == "round":
        return {"scale": scale, "values": w.to(out)}
    x, dy = s["x"].float(), s["dy"].float()
    return {"y": (x @ w.t()).to(out), "dx": (dy @ w).to(out), "dw": (dy.t() @ x).to(out)}


def _kernels(s):
    import paper_2504_17785_amd as slz

    kind = s["kind"]
    if kind == "clip":
        return [slz.clip_by_norm(s["g"], 1.0, EPS, out=s["out"])] + s["buckets"]
    group = s["group"]
    if kind == "linear":
        return {"y": slz.linear_i4(s["x"], s["q"], s["scale"], group)}
    q, scale = slz.quantize_i4(s["w"], group)
    if kind == "round":
        return {"scale": scale, "values": slz.values_i4(q, scale, s["w"].shape[1], group, s["dtype"])}
    y = slz.linear_i4(s["x"], q, scale, group)
    dx, dw = slz.linear_i4_grad(s["dy"], s["x"], q, scale, group)
    return {"y": y, "dx": dx, "dw": dw}


def run(state):
    return _kernels(state) if own else _plain(state)


def work(case):
    kind = case["kind"]
    if kind == "clip":
        size = sum(math.prod(s) * (4 if case["dtype"] == "f32" or (bias and case["dtype"] == "mixed") else 2) for s, bias in _tensors(case))
        count = sum(math.prod(s) for s, _ in _tensors(case))
        return {"bytes": 2 * size, "flops": 3 * count}
    M, K, N, e = case["tokens"], case["inner"], case["outer"], BYTES[case["dtype"]]
    weights = N * ((K + 1) // 2) + 4 * N * ((K + case["group"] - 1) // case["group"])
    if kind == "linear":
        return {"bytes": e * M * (K + N) + weights, "flops": 2 * M * N * K}
    if kind == "round":
        return {"bytes": 2 * e * N * K + weights, "flops": 4 * N * K}
    return {"bytes": 2 * e * (M * K + N * K + M * N), "flops": 6 * M * N * K}


def exact(case, seed):
    s, wide = prepare(case, seed), torch.float64
    kind = s["kind"]
    if kind == "clip":
        norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g.to(wide)) for g in s["g"]]))
        by = 1.0 / (norm + EPS)
        flat = {}
        for g in s["g"]:
            values = flat.setdefault(g.dtype, [])
            values.append(g.to(wide).flatten() * (by if by < 1 else 1.0))
            values.append(torch.zeros(-g.numel() % 64, dtype=wide, device="cuda"))
        return [norm] + [torch.cat(values) for values in flat.values()]
    group = s["group"]
    if kind == "linear":
        n, k = s["q"].shape[0], s["x"].shape[1]
        words = s["q"].contiguous().view(torch.int32).to(torch.int64) & 0xffffffff
        w = torch.empty((n, words.shape[1] * 8), dtype=wide, device="cuda")
        for j in range(4):
            for step in range(4):
                for e in range(8):
                    code = (words[:, 4 * j + step::16] >> (8 * (e % 4) + 4 * (e // 4))) & 15
                    w[:, 32 * step + 8 * j + e::128] = (code % 8) * (1 - 2 * (code // 8))
        w = w[:, :k]
        for i in range(s["scale"].shape[1]):
            w[:, i * group:(i + 1) * group] *= s["scale"][:, i:i + 1].to(wide)
        return {"y": torch.mm(s["x"].to(wide), w.t())}
    w, scales = s["w"].to(wide), []
    values = torch.empty_like(w)
    for at in range(0, w.shape[1], group):
        part = w[:, at:at + group]
        top = part.abs().max(dim=1, keepdim=True).values
        values[:, at:at + group] = torch.where(top > 0, torch.round(part * 7 / top) * (top / 7), 0.0)
        scales.append(top / 7)
    if kind == "round":
        return {"scale": torch.cat(scales, dim=1), "values": values}
    x, dy = s["x"].to(wide), s["dy"].to(wide)
    return {"y": torch.mm(x, values.t()), "dx": torch.mm(dy, values), "dw": torch.mm(dy.t(), x)}
