"""Cases and plain forms of the operators of training and running a network in the clear (include/silenzio_clear.h).

A case is a dict of plain values with a "kind":
  linear   x [tokens][inner] floating -> rows quantised to 8 bits -> product with 8-bit weights [outer][inner] that the program keeps
  product  8-bit a [tokens][inner] and b [outer][inner], a scale for each row of either -> their product
  train    one step of such a layer: x and w quantised, y, and with dy the gradients of x and w
  score    softmax cross entropy of h [tokens][inner] against w [outer][inner] (outer: the vocabulary): loss and log-sum of each token
  loss     the same with the gradients of h and w
  update   a batch of gradients [tokens][inner] orthogonalised by Newton-Schulz products
"dtype" is the type of the floating inputs and outputs; "slack" is how many elements the rows of the first input lie further apart
than they are long.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
IGNORED = -100
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS, EPS = 5, 1e-7


def _case(name, kind, tokens, inner, outer=0, dtype="bf16", slack=0, batch=1):
    return dict(name=name, kind=kind, tokens=tokens, inner=inner, outer=outer, dtype=dtype, slack=slack, batch=batch)


def listed():
    return [
        # one token through a layer whose weights stay in 8 bits: a step of serving
        _case("linear_1x4096x8192", "linear", 1, 4096, 8192),
        # the first layer of the library's MLP (784 -> 128) on a mini-batch of 32 images
        _case("linear_32x784x128", "linear", 32, 784, 128, "f32"),
        # matrices that are quantised already, no size a multiple of anything
        _case("product_777x1555x1001", "product", 777, 1555, 1001, "f16", 5),
        # a training step of a square layer: quantise both, forward, both gradients
        _case("train_4096x4096x4096", "train", 4096, 4096, 4096),
        # a long prompt, or a large batch, through a wide layer
        _case("linear_8192x8192x8192", "linear", 8192, 8192, 8192, "f16"),
        # a classifier's head of 10 classes on a mini-batch of 32: launches and latency
        _case("loss_32x128x10", "loss", 32, 128, 10, "f32"),
        # the log-likelihoods of a few tokens: the vocabulary's weights are read once
        _case("score_8x2048x65536", "score", 8, 2048, 65536),
        # a training step's loss on a batch of ragged sequences, some tokens padding, an odd vocabulary
        _case("loss_1003x768x50021", "loss", 1003, 768, 50021, "f16", 8),
        # the same at the size of a large model's step
        _case("loss_4096x4096x131072", "loss", 4096, 4096, 131072),
        # the gradient of the library's 784 -> 128 layer
        _case("update_128x784", "update", 128, 784),
        # the gradients of six layers of one shape, taller than wide
        _case("update_6x1000x500", "update", 1000, 500, dtype="f16", batch=6),
        # one large layer
        _case("update_4096x8192", "update", 4096, 8192),
    ]


def _log(rng, low, high):
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    kind = rng.choice(("linear", "linear", "product", "train", "score", "loss", "loss", "update", "update"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    slack = rng.choice((0, 0, 1, 8))
    while True:
        if kind in ("score", "loss"):
            c = _case("", kind, _log(rng, 1, 4096), _log(rng, 32, 4096), _log(rng, 2, 131072), dtype, slack)
        elif kind == "update":
            c = _case("", kind, _log(rng, 8, 8192), _log(rng, 8, 8192), 0, dtype, slack, rng.choice((1, 1, 2, 5, 16)))
        else:
            c = _case("", kind, _log(rng, 1, 8192), _log(rng, 32, 8192), _log(rng, 32, 8192), dtype, slack)
        # no more than the largest listed case of its kind, and memory for three states
        if work(c)["flops"] <= (1.4e13 if kind in ("score", "loss") else 4.2e12) and c["batch"] * c["tokens"] * c["inner"] <= 2 ** 27:
            del c["name"]
            return c


def _rows(gen, rows, cols, dtype, slack, std):
    """Values of a row-major matrix whose rows lie `slack` elements further apart than they are long."""
    t = torch.randn((*rows, cols + slack), device="cuda", generator=gen) * std
    return t.to(TYPES[dtype])[..., :cols]


def _int8(gen, rows, cols, slack=0):
    t = (torch.randn((rows, cols + slack), device="cuda", generator=gen) * 32).round().clamp(-127, 127)
    return t.to(torch.int8)[:, :cols]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind, M, K, N, dtype, slack = (case[k] for k in ("kind", "tokens", "inner", "outer", "dtype", "slack"))
    s = {"kind": kind, "dtype": TYPES[dtype]}
    if kind in ("linear", "train"):
        # activations after a norm: unit variance, a few channels larger
        s["x"] = _rows(gen, (M,), K, dtype, slack, 1.0)
        s["x"][:, ::61] *= 4
    if kind == "linear":
        s["w"] = _int8(gen, N, K)
    if kind == "product":
        s["a"], s["w"] = _int8(gen, M, K, slack), _int8(gen, N, K, slack)
        s["a_scale"] = torch.rand(M, device="cuda", generator=gen) * 0.05 + 0.01
    if kind in ("linear", "product"):
        s["w_scale"] = (torch.rand(N, device="cuda", generator=gen) + 0.5) / (32 * math.sqrt(K))
    if kind == "train":
        s["w"] = _rows(gen, (N,), K, dtype, 0, 1 / math.sqrt(K))
        s["dy"] = _rows(gen, (M,), N, dtype, 0, 1 / math.sqrt(N))
    if kind in ("score", "loss"):
        # hidden states after a norm; logits of a spread of 2, a third of the labels among the likelier words, some tokens padding
        s["x"] = _rows(gen, (M,), K, dtype, slack, 1.0)
        s["w"] = _rows(gen, (N,), K, dtype, 0, 2 / math.sqrt(K))
        labels = torch.randint(0, N, (M,), device="cuda", generator=gen)
        t = torch.arange(M, device="cuda")
        near = (s["x"][::3].float() @ s["w"][:4096].float().t()).argmax(1)
        labels[::3] = near
        labels[t % 8 == 5] = IGNORED
        s["labels"] = labels
        # the mean over the tokens that count
        s["dloss"] = torch.full((M,), 1.0 / max(1, M - (M + 2) // 8), device="cuda")
    if kind == "update":
        # a gradient: a few strong directions over noise
        g = torch.randn((case["batch"], M, K + slack), device="cuda", generator=gen)
        u = torch.randn((case["batch"], M, 4), device="cuda", generator=gen)
        v = torch.randn((case["batch"], 4, K + slack), device="cuda", generator=gen)
        s["g"] = ((g + torch.matmul(u, v)) * 1e-3).to(TYPES[dtype])[:, :, :K]
    return s


def _quantised(x):
    """Rows to whole numbers in [-127, 127], in the input's precision, and a scale for each."""
    top = x.abs().amax(1)
    q = torch.round(x * torch.where(top > 0, 127.0 / top, torch.zeros_like(top))[:, None]).clamp(-127, 127)
    return q, top / 127.0


def _plain(s):
    kind, out = s["kind"], s["dtype"]
    if kind in ("linear", "product"):
        a, sa = _quantised(s["x"].float()) if kind == "linear" else (s["a"].float(), s["a_scale"])
        return {"y": (a @ s["w"].float().t() * (sa[:, None] * s["w_scale"][None, :])).to(out)}
    if kind == "train":
        a, sa = _quantised(s["x"].float())
        b, sb = _quantised(s["w"].float())
        a_value, b_value, dy = a * sa[:, None], b * sb[:, None], s["dy"].float()
        return {"y": (a @ b.t() * (sa[:, None] * sb[None, :])).to(out), "dx": (dy @ b_value).to(out), "dw": (dy.t() @ a_value).to(out)}
    if kind in ("score", "loss"):
        h, w, labels = s["x"].float(), s["w"].float(), s["labels"]
        z = h @ w.t()
        top = z.amax(1, keepdim=True)
        lse = (torch.log(torch.exp(z - top).sum(1, keepdim=True)) + top)[:, 0]
        counts = labels != IGNORED
        at = torch.where(counts, labels, 0)[:, None]
        loss = torch.where(counts, lse - z.gather(1, at)[:, 0], torch.zeros_like(lse))
        if kind == "score":
            return {"loss": loss, "lse": lse}
        g = torch.exp(z - lse[:, None])
        g.scatter_add_(1, at, torch.full_like(lse, -1.0)[:, None])
        g = g * torch.where(counts, s["dloss"], torch.zeros_like(lse))[:, None]
        return {"loss": loss, "lse": lse, "dh": (g @ w).to(out), "dw": (g.t() @ h).to(out)}
    a, b, c = COEFFICIENTS
    x = s["g"].float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / (torch.sqrt((x * x).sum((1, 2), keepdim=True)) + EPS)
    for _ in range(STEPS):
        gram = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * gram + c * torch.matmul(gram, gram), x)
    return {"update": (x.transpose(1, 2).contiguous() if tall else x).to(out)}


def _kernels(s):
    import paper_2504_17785_amd as slz

    kind, out = s["kind"], s["dtype"]
    if kind == "linear":
        return {"y": slz.linear_i8(s["x"], s["w"], s["w_scale"])}
    if kind == "product":
        return {"y": slz.matmul_i8(s["a"], s["a_scale"], s["w"], s["w_scale"], out)}
    if kind == "train":
        a, sa = slz.quantize_i8(s["x"])
        b, sb = slz.quantize_i8(s["w"])
        y = slz.matmul_i8(a, sa, b, sb, out)
        dx, dw = slz.matmul_i8_grad(s["dy"], a, sa, b, sb)
        return {"y": y, "dx": dx, "dw": dw}
    if kind in ("score", "loss"):
        loss, lse = slz.linear_ce(s["x"], s["w"], s["labels"], ignore_index=IGNORED)
        if kind == "score":
            return {"loss": loss, "lse": lse}
        dh, dw = slz.linear_ce_grad(s["x"], s["w"], s["labels"], lse, s["dloss"], ignore_index=IGNORED)
        return {"loss": loss, "lse": lse, "dh": dh, "dw": dw}
    return {"update": slz.orthogonalize(s["g"], STEPS, COEFFICIENTS, EPS)}


def run(state):
    return _kernels(state) if own else _plain(state)


def work(case):
    kind, M, K, N, e = case["kind"], case["tokens"], case["inner"], case["outer"], BYTES[case["dtype"]]
    if kind == "linear":
        return {"bytes": e * M * K + N * K + 4 * N + e * M * N, "flops": 2 * M * N * K}
    if kind == "product":
        return {"bytes": M * K + N * K + 4 * (M + N) + e * M * N, "flops": 2 * M * N * K}
    if kind == "train":
        return {"bytes": 2 * e * (M * K + N * K + M * N), "flops": 6 * M * N * K}
    if kind == "score":
        return {"bytes": e * (M + N) * K + 16 * M, "flops": 2 * M * N * K}
    if kind == "loss":
        return {"bytes": 2 * e * (M + N) * K + 20 * M, "flops": 6 * M * N * K}
    m, n = min(M, K), max(M, K)
    # X X^T and A A are symmetric: half of each
    return {"bytes": 2 * e * case["batch"] * m * n, "flops": case["batch"] * STEPS * (3 * m * m * n + m ** 3)}


def exact(case, seed):
    s, wide = prepare(case, seed), torch.float64
    kind = s["kind"]

    def whole(x):
        x = x.to(wide)
        most = x.abs().max(dim=1, keepdim=True).values
        step = most / 127
        return torch.where(most > 0, torch.round(x / torch.where(most > 0, step, torch.ones_like(step))), torch.zeros_like(x)) * step

    if kind in ("linear", "product"):
        left = whole(s["x"]) if kind == "linear" else s["a"].to(wide) * s["a_scale"].to(wide).unsqueeze(1)
        return {"y": torch.mm(left, (s["w"].to(wide) * s["w_scale"].to(wide).unsqueeze(1)).t())}
    if kind == "train":
        left, right, dy = whole(s["x"]), whole(s["w"]), s["dy"].to(wide)
        return {"y": torch.mm(left, right.t()), "dx": torch.mm(dy, right), "dw": torch.mm(dy.t(), left)}
    if kind in ("score", "loss"):
        h, w, labels = s["x"].to(wide), s["w"].to(wide), s["labels"]
        z = torch.mm(h, w.t())
        lse = torch.logsumexp(z, dim=1)
        kept = torch.nonzero(labels != IGNORED).squeeze(1)
        loss = torch.zeros(len(labels), dtype=wide, device=z.device)
        loss[kept] = lse[kept] - z[kept, labels[kept]]
        if kind == "score":
            return {"loss": loss, "lse": lse}
        z.sub_(lse.unsqueeze(1)).exp_()
        z[kept, labels[kept]] -= 1
        weight = torch.zeros_like(lse)
        weight[kept] = s["dloss"].to(wide)[kept]
        z.mul_(weight.unsqueeze(1))
        return {"loss": loss, "lse": lse, "dh": torch.mm(z, w), "dw": torch.mm(z.t(), h)}
    a, b, c = COEFFICIENTS
    done = []
    for g in s["g"].to(wide):
        x = g.t() if g.shape[0] > g.shape[1] else g
        x = x / (torch.linalg.vector_norm(x) + EPS)
        one = torch.eye(x.shape[0], dtype=wide, device=x.device)
        for _ in range(STEPS):
            gram = torch.mm(x, x.t())
            x = torch.mm(a * one + torch.mm(gram, b * one + c * gram), x)
        done.append(x.t() if g.shape[0] > g.shape[1] else x)
    return {"update": torch.stack(done)}
