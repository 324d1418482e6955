"""The operators of include/silenzio_clear.h against their formulas in 64 bits.

U is a type's unit roundoff (half the distance of 1 and the next number).  A sum of n products in 32 bits is off by at most (n + 2) 2^-24 of
the sum of their magnitudes; an operand rounded to a type adds U of it; three bf16 carry a 32-bit number, and the products of them that are
left out are below 2^-21 of the magnitudes."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}     # smallest numbers
TYPES = (torch.float32, torch.bfloat16, torch.float16)
IGNORED = -100
WIDE = torch.float64


@pytest.fixture(scope="module")
def slz():
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a GPU: torch.cuda.is_available() is False")
    import paper_2504_17785_amd as m
    m.lib()
    return m


def randn(shape, seed, dtype=torch.float32, slack=0, skip=0, std=1.0):
    """Normal values; rows `slack` elements further apart than they are long, the first one `skip` elements into its storage."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randn((*shape[:-1], shape[-1] + slack + skip), device="cuda", generator=gen) * std
    return t.to(dtype)[..., skip:skip + shape[-1]]


def int8(shape, seed, slack=0, skip=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randint(-128, 128, (shape[0], shape[1] + slack + skip), device="cuda", generator=gen, dtype=torch.int8)
    return t[:, skip:skip + shape[1]]


def scales(n, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.rand(n, device="cuda", generator=gen) * 0.02 + 0.001


def inside(got, want, bound, what=""):
    """Every element of got is as near to want (64 bits) as bound says, and NaN where want is."""
    got = got.to(WIDE)
    assert got.shape == want.shape, what
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    off = torch.nan_to_num((got - want).abs() - bound)
    assert not (off > 0).any(), "%s: %g over a bound of %g" % (what, off.max().item(), bound.max().item() if torch.is_tensor(bound) else bound)


# ---- 8-bit integers -----------------------------------------------------------------------------------------------------------
def quantised(x):
    """The definition in 32 bits, on the host."""
    x = x.float().cpu().numpy()
    top = np.abs(x).max(axis=1, initial=0).astype(np.float32)
    with np.errstate(all="ignore"):
        inv = np.where(top > 0, np.float32(1) / top * np.float32(127), np.float32(0)).astype(np.float32)
        q = np.rint(x * inv[:, None])
    return q.astype(np.int8), (top / np.float32(127)).astype(np.float32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,slack", [(1, 1, 0), (3, 7, 2), (5, 64, 0), (2, 1000, 1), (33, 784, 0), (4, 4096, 8), (7, 8192, 0), (2, 20001, 3), (70000, 5, 0)])
def test_quantize_is_the_definition(slz, dtype, rows, cols, slack):
    x = randn((rows, cols), rows + cols, dtype, slack)
    x[rows // 2] *= 1e-3
    q, scale = slz.quantize_i8(x)
    want_q, want_scale = quantised(x)
    assert np.array_equal(q.cpu().numpy(), want_q)
    assert np.array_equal(scale.cpu().numpy(), want_scale)


def test_quantize_of_rows_without_a_scale(slz):
    for cols in (9, 3000):
        x = randn((6, cols), 1)
        x[1] = 0
        x[2, 3] = float("inf")
        x[3, cols - 1] = float("nan")
        x[4] *= 1e-38 / x[4].abs().max()           # 127 / top is not a 32-bit number
        x[5] = -0.0
        q, scale = slz.quantize_i8(x)
        assert (q[1:4] == 0).all() and (q[5] == 0).all()
        assert scale[1] == 0 and scale[5] == 0 and torch.isnan(scale[2:4]).all()
        assert q[4].abs().max() == 127
        back = q[4].to(WIDE) * scale[4].to(WIDE)
        # half a step, the scale's own rounding (it is a subnormal number) and that of x * inv
        inside(back, x[4].to(WIDE), 0.5001 * 1e-38 / 127 + 128 * 2.0 ** -149, "tiny")
    q, scale = slz.quantize_i8(torch.empty((3, 0), device="cuda"))
    assert q.shape == (3, 0) and (scale == 0).all()
    q, scale = slz.quantize_i8(torch.empty((0, 5), device="cuda"))
    assert q.shape == (0, 5) and scale.shape == (0,)


PRODUCTS = [(1, 1, 1), (1, 5, 16), (2, 3, 31), (1, 128, 784), (1, 4096, 1024), (3, 777, 130), (16, 256, 4096), (17, 100, 64), (32, 128, 784), (33, 65, 129),
            (64, 1000, 4099), (127, 129, 127), (128, 128, 128), (130, 257, 255), (257, 300, 1000), (500, 1100, 70), (1030, 520, 33), (5, 2, 100001), (700, 40, 20000)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_matmul_i8_is_exact_up_to_its_roundings(slz, dtype, m, n, k):
    slack = (m + n + k) % 3
    a, b = int8((m, k), 1, slack), int8((n, k), 2, 2 * slack)
    a[0, 0], b[0, 0] = -128, -128
    sa, sb = scales(m, 3), scales(n, 4)
    y = slz.matmul_i8(a, sa, b, sb, dtype)
    assert y.dtype == dtype
    want = (a.cpu().to(WIDE) @ b.cpu().to(WIDE).t()).cuda() * sa.to(WIDE)[:, None] * sb.to(WIDE)[None, :]
    # the sum to 32 bits, the scales' product, their product, and the type's own rounding
    inside(y, want, want.abs() * (3.01 * 2.0 ** -24 + 1.01 * U[dtype]) + LEAST[dtype], "y")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_linear_i8_is_quantize_then_matmul(slz, dtype, m, n, k):
    x = randn((m, k), 5, dtype, slack=(m + n) % 3)
    w, sw = int8((n, k), 6, slack=k % 2), scales(n, 7)
    if m > 2:
        x[1] = 0
        x[2, k // 2] = float("nan")
    y = slz.linear_i8(x, w, sw)
    q, sx = slz.quantize_i8(x)
    assert torch.equal(y.nan_to_num(nan=7.0), slz.matmul_i8(q, sx, w, sw, dtype).nan_to_num(nan=7.0))
    if m > 2:
        assert (y[1] == 0).all() and torch.isnan(y[2]).all()


def test_matmul_i8_at_any_address(slz):
    for skip in (1, 3, 16):
        a, b = int8((40, 208), 1, 0, skip), int8((50, 208), 2, 5, skip)
        sa, sb = scales(40, 3), scales(50, 4)
        y = slz.matmul_i8(a, sa, b, sb, torch.float32)
        assert torch.equal(y, slz.matmul_i8(a.contiguous(), sa, b.contiguous(), sb, torch.float32))


def test_matmul_i8_without_elements(slz):
    one = scales(3, 1)
    y = slz.matmul_i8(torch.empty((3, 0), dtype=torch.int8, device="cuda"), one, torch.empty((3, 0), dtype=torch.int8, device="cuda"), one)
    assert y.shape == (3, 3) and (y == 0).all()
    assert slz.linear_i8(torch.empty((0, 8), device="cuda"), int8((3, 8), 1), one).shape == (0, 3)
    assert slz.linear_i8(torch.empty((3, 8), device="cuda"), int8((0, 8), 1), one[:0]).shape == (3, 0)


GRADS = [(1, 1, 1), (1, 128, 784), (3, 7, 5), (32, 128, 784), (65, 33, 130), (128, 128, 128), (130, 257, 255), (300, 1000, 200), (1000, 70, 513), (17, 2050, 64)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", GRADS)
def test_matmul_i8_grad_is_the_formula(slz, dtype, m, n, k):
    dy = randn((m, n), 8, dtype, slack=(m + k) % 3)
    a, b = int8((m, k), 9, slack=m % 2), int8((n, k), 10)
    sa, sb = scales(m, 11), scales(n, 12) * 1e-3
    da, db = slz.matmul_i8_grad(dy, a, sa, b, sb)
    A, B, D = a.cpu().to(WIDE) * sa.cpu().to(WIDE)[:, None], b.cpu().to(WIDE) * sb.cpu().to(WIDE)[:, None], dy.cpu().to(WIDE)
    for got, want, size, terms, largest in ((da, D @ B, D.abs() @ B.abs(), n, sb.max()), (db, D.t() @ A, D.abs().t() @ A.abs(), m, sa.max())):
        # values rounded to the type (f32: in three pieces), sums, result; f16 values below 2^-14 of the largest scale lose bits
        bound = size * ((1.01 * U[dtype] if dtype != torch.float32 else 2.0 ** -21) + (terms + 4) * 2.0 ** -24) + want.abs() * 1.01 * U[dtype] + LEAST[dtype]
        if dtype == torch.float16:
            bound = bound + 2.0 ** -24 * largest.item() * 2 * terms * D.abs().max()
        inside(got, want.cuda(), bound.cuda(), "gradient")
    only_a, none = slz.matmul_i8_grad(dy, a, sa, b, sb, need_b=False)
    assert none is None and torch.equal(only_a, da)
    none, only_b = slz.matmul_i8_grad(dy, a, sa, b, sb, need_a=False)
    assert none is None and torch.equal(only_b, db)


def test_matmul_i8_grad_against_differences(slz):
    # y is linear in either matrix: <dy, y(a + d) - y(a)> = <da, a_scale d>, exactly but for roundings
    m, n, k = 40, 30, 50
    a, b, d = int8((m, k), 1) // 4, int8((n, k), 2) // 4, int8((m, k), 3) // 4
    e = int8((n, k), 4) // 4
    sa, sb, dy = scales(m, 5), scales(n, 6), randn((m, n), 7)
    da, db = slz.matmul_i8_grad(dy, a, sa, b, sb)

    def y(a, b):
        return slz.matmul_i8(a, sa, b, sb, torch.float32).to(WIDE)

    for diff, grad, step in ((y(a + d, b) - y(a, b), da, d.to(WIDE) * sa.to(WIDE)[:, None]), (y(a, b + e) - y(a, b), db, e.to(WIDE) * sb.to(WIDE)[:, None])):
        left, right = (dy.to(WIDE) * diff).sum(), (grad.to(WIDE) * step).sum()
        size = (dy.to(WIDE).abs() * (y(a, b).abs() + y(a + d, b).abs() + y(a, b + e).abs())).sum() + (grad.to(WIDE).abs() * step.abs()).sum() * 4
        assert abs(left - right) < size * 64 * 2.0 ** -21


# ---- cross entropy ---------------------------------------------------------------------------------------------------------------
def ce_reference(h, w, labels, ignore=IGNORED):
    z = h.to(WIDE) @ w.to(WIDE).t().contiguous()
    lse = torch.logsumexp(z, 1)
    counts = labels != ignore
    bad = counts & ((labels < 0) | (labels >= w.shape[0]))
    at = torch.where(counts & ~bad, labels, 0)
    loss = torch.where(counts, lse - z.gather(1, at[:, None])[:, 0], torch.zeros_like(lse))
    loss[bad] = float("nan")
    return z, lse, loss, counts, bad, at


def ce_bounds(h, w):
    """What z may be off by, per token: products summed in 32 bits, for f32 without the smallest of the pieces' products."""
    size = (h.to(WIDE).abs() @ w.to(WIDE).abs().t().contiguous()).amax(1)
    return size * ((h.shape[1] + 4) * 2.0 ** -24 + (2.0 ** -21 if h.dtype == torch.float32 else 0.0))


def check_ce(slz, h, w, labels, dloss, ignore=IGNORED):
    dtype = h.dtype
    z, lse, loss, counts, bad, at = ce_reference(h, w, labels, ignore)
    ez = ce_bounds(h, w)
    got_loss, got_lse = slz.linear_ce(h, w, labels, ignore)
    # exp and log in 32 bits: 2^-18 covers the arguments' rounding at a distance of 60 from the maximum and the sums
    near = 2 * ez + 2.0 ** -18 + lse.abs() * 2.0 ** -22
    inside(got_lse, lse, near, "lse")
    inside(got_loss, loss, near + ez + loss.abs().nan_to_num() * 2.0 ** -22, "loss")
    assert (got_loss[~counts] == 0).all()
    dh, dw = slz.linear_ce_grad(h, w, labels, got_lse, dloss, ignore)
    p = torch.exp(z - lse[:, None])
    one = torch.zeros_like(p)
    rows = torch.nonzero(counts & ~bad)[:, 0]
    one[rows, at[rows]] = 1
    by = torch.where(counts, dloss.to(WIDE), torch.zeros_like(lse))
    by[bad] = float("nan")
    g = (p - one) * by[:, None]
    # p from z and lse, exp in 32 bits; p - 1 and the product with dloss; the type of g (f16: 2^-24 2^-14 of twice the largest dloss at least)
    eg = by.abs()[:, None] * p * (ez + near + 2.0 ** -18)[:, None] + g.abs() * (1.01 * U[dtype] if dtype != torch.float32 else 2.0 ** -21)
    eg = eg + by.abs()[:, None] * 2.0 ** -23
    if dtype == torch.float16:
        eg = eg + 2.0 ** -38 * 2 * dloss.abs().max()
    for got, want, size, off, terms in ((dh, g @ w.to(WIDE), g.abs() @ w.to(WIDE).abs(), eg @ w.to(WIDE).abs(), w.shape[0]),
                                        (dw, g.t().contiguous() @ h.to(WIDE), g.abs().t().contiguous() @ h.to(WIDE).abs(), eg.t().contiguous() @ h.to(WIDE).abs(), h.shape[0])):
        bound = off + size * ((terms + 4) * 2.0 ** -24 + (2.0 ** -21 if dtype == torch.float32 else 0.0)) + want.abs() * 1.01 * U[dtype] + LEAST[dtype]
        inside(got, want, bound, "gradient")
    return got_loss, got_lse, dh, dw


def ce_inputs(tokens, inner, vocab, dtype, seed, slack=0, skip=0):
    h = randn((tokens, inner), seed, dtype, slack, skip)
    w = randn((vocab, inner), seed + 1, dtype, slack, skip, 2 / inner ** 0.5)
    gen = torch.Generator(device="cuda").manual_seed(seed + 2)
    labels = torch.randint(0, vocab, (tokens,), device="cuda", generator=gen)
    dloss = torch.rand(tokens, device="cuda", generator=gen) - 0.3
    return h, w, labels, dloss


LOSSES = [(1, 1, 1), (1, 64, 2), (8, 8, 3), (5, 128, 10), (32, 128, 10), (1, 512, 5000), (16, 256, 1000), (33, 40, 129), (128, 64, 128), (130, 72, 257), (200, 264, 1025),
          (515, 128, 3001), (3, 1000, 40), (129, 17, 130),
          (33, 128, 10), (300, 100, 16), (100, 512, 16), (9000, 20, 7), (100, 500, 32), (100, 513, 32), (5, 8192, 2), (70, 2047, 8), (1100, 3000, 40)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,inner,vocab", LOSSES)
def test_linear_ce_is_the_formula(slz, dtype, tokens, inner, vocab):
    h, w, labels, dloss = ce_inputs(tokens, inner, vocab, dtype, 20, slack=(tokens + vocab) % 3)
    labels[::7] = vocab - 1
    labels[3::5] = IGNORED
    check_ce(slz, h, w, labels, dloss)


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_ce_labels(slz, dtype):
    h, w, labels, dloss = ce_inputs(40, 48, 300, dtype, 30)
    check_ce(slz, h, w, torch.full_like(labels, IGNORED), dloss)           # no token counts: zero losses, zero gradients
    dh, dw = slz.linear_ce_grad(h, w, torch.full_like(labels, IGNORED), torch.zeros_like(dloss), dloss)
    assert (dh == 0).all() and (dw == 0).all()
    check_ce(slz, h, w, torch.where(labels % 3 == 0, 7, labels), dloss, ignore=7)          # a word of the vocabulary as the one to ignore
    loss, _ = slz.linear_ce(h, w, torch.where(labels % 2 == 0, 300, -1), -1)
    assert torch.equal(torch.isnan(loss), labels % 2 == 0) and (loss[labels % 2 == 1] == 0).all()
    outside = labels.clone()
    outside[4] = 300
    outside[9] = -2
    loss, lse = slz.linear_ce(h, w, outside)
    assert torch.isnan(loss[[4, 9]]).all() and torch.isfinite(loss).sum() == 38
    dh, _ = slz.linear_ce_grad(h, w, outside, lse, dloss)
    assert torch.isnan(dh[[4, 9]]).all() and torch.isfinite(dh).all(1).sum() == 38


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_ce_of_large_and_missing_values(slz, dtype):
    h, w, labels, dloss = ce_inputs(40, 64, 300, dtype, 40)
    check_ce(slz, (h * 16).contiguous(), (w * 4).contiguous(), labels, dloss)       # logits of some hundred: one word has it all
    check_ce(slz, h * 0, w, labels, dloss)
    h[5, 3] = float("nan")
    h[6, 3] = float("inf")
    loss, lse = slz.linear_ce(h, w, labels)
    gone = torch.zeros(40, dtype=torch.bool, device="cuda")
    gone[5:7] = True
    assert torch.equal(torch.isnan(loss), gone) and torch.equal(torch.isnan(lse), gone)
    # a word that no token can be: z = -inf adds nothing
    h, w, labels, dloss = ce_inputs(40, 64, 300, dtype, 41)
    h[:, 0] = 1
    w[17, 0] = w[200, 0] = float("-inf")
    labels[labels == 17] = 18
    labels[labels == 200] = 201
    loss, lse = slz.linear_ce(h, w, labels)
    keep = [i for i in range(300) if i not in (17, 200)]
    if dtype != torch.float32:                                      # in three pieces an infinity meets zeros of the others
        inside(lse, torch.logsumexp(h.to(WIDE) @ w[keep].to(WIDE).t().contiguous(), 1), ce_bounds(h, w[keep]) * 2 + 2.0 ** -17, "lse")
        assert torch.isfinite(loss).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_ce_at_any_address(slz, dtype):
    h, w, labels, dloss = ce_inputs(50, 64, 400, dtype, 50, slack=5, skip=1)
    first = check_ce(slz, h, w, labels, dloss)
    again = check_ce(slz, h.contiguous(), w.contiguous(), labels, dloss)
    for x, y in zip(first, again):
        assert torch.equal(x, y)


def test_linear_ce_in_several_pieces_of_the_vocabulary(slz):
    # 16384 tokens: a piece's gradient of the logits is held for 8192 words (bf16)
    tokens, inner, vocab = 16384, 32, 20001
    h, w, labels, dloss = ce_inputs(tokens, inner, vocab, torch.bfloat16, 60)
    loss, lse = slz.linear_ce(h, w, labels)
    dh, dw = slz.linear_ce_grad(h, w, labels, lse, dloss)
    # each token's gradient does not depend on the others
    rows = torch.arange(0, tokens, 331, device="cuda")
    few = check_ce(slz, h[rows].contiguous(), w, labels[rows].contiguous(), dloss[rows].contiguous())
    assert torch.equal(few[0], loss[rows]) and torch.equal(few[1], lse[rows])
    want = few[2].to(WIDE)
    # the same sums in another order, and both rounded once
    assert ((dh[rows].to(WIDE) - want).norm() <= 2 * U[torch.bfloat16] * want.norm())
    sums = dw.to(WIDE).sum(0)
    z = torch.exp(h.float() @ w.float().t() - lse[:, None])
    z[torch.arange(tokens, device="cuda"), labels] -= 1
    z *= dloss[:, None]
    want = z.t().contiguous() @ h.float()
    assert ((dw.float() - want).norm() <= 3 * U[torch.bfloat16] * want.norm()), sums


@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_of_any_scale(slz, dtype):
    # f16 holds what is relative to the largest: gradients of 1e-30 or 1e4, and an ignored token's that is not a number
    h, w, labels, dloss = ce_inputs(40, 64, 300, dtype, 42)
    labels[7] = IGNORED
    for scale in (1e-3, 1e3):
        by = dloss * scale
        check_ce(slz, h, w, labels, by)
        by[7] = float("inf")
        lse = slz.linear_ce(h, w, labels)[1]
        first = slz.linear_ce_grad(h, w, labels, lse, by)
        by[7] = 0
        second = slz.linear_ce_grad(h, w, labels, lse, by)
        assert torch.equal(first[0], second[0]) and torch.equal(first[1], second[1])
    if dtype == torch.float32:
        dh, dw = slz.linear_ce_grad(h, w, labels, lse, dloss * 1e-30)
        one, two = slz.linear_ce_grad(h, w, labels, lse, dloss)
        for got, want in ((dh, one), (dw, two)):
            assert ((got.to(WIDE) * 1e30 - want.to(WIDE)).norm() <= 2.0 ** -20 * want.to(WIDE).norm())


def test_a_loss_has_the_same_bits_alone_and_among_others(slz):
    for dtype in TYPES:
        for inner, vocab in ((64, 10), (72, 700), (520, 5000)):
            h, w, labels, _ = ce_inputs(900, inner, vocab, dtype, 43)
            loss, lse = slz.linear_ce(h, w, labels)
            for part in (slice(0, 1), slice(5, 12), slice(100, 250), slice(3, 900, 7)):
                a, b = slz.linear_ce(h[part].contiguous(), w, labels[part].contiguous())
                assert torch.equal(a, loss[part]) and torch.equal(b, lse[part])


def test_linear_ce_past_four_gib(slz):
    tokens, inner, vocab = 3, 4096, 560000
    h = randn((tokens, inner), 1, torch.bfloat16)
    w = torch.empty((vocab, inner), dtype=torch.bfloat16, device="cuda")
    for v in range(0, vocab, 70000):
        w[v:v + 70000] = randn((70000, inner), 2 + v, torch.bfloat16, std=2 / 64)
    labels = torch.tensor([vocab - 1, 540000, 7], device="cuda")
    dloss = torch.tensor([0.5, -1.0, 2.0], device="cuda")
    z = torch.cat([h.float() @ w[v:v + 70000].float().t() for v in range(0, vocab, 70000)], 1).to(WIDE)
    loss, lse = slz.linear_ce(h, w, labels)
    want = torch.logsumexp(z, 1)
    # both products in 32 bits: 4096 terms each
    bound = 2 * 4100 * 2.0 ** -24 * (h.float().abs() @ w[:2000].float().abs().t()).max().item() * 1.5 + 2.0 ** -17
    inside(lse, want, bound, "lse")
    inside(loss, want - z.gather(1, labels[:, None])[:, 0], 2 * bound, "loss")
    dh, dw = slz.linear_ce_grad(h, w, labels, lse, dloss)
    g = torch.exp(z - want[:, None])
    g[torch.arange(3, device="cuda"), labels] -= 1
    g *= dloss[:, None]
    for v in (0, 262144, 524288, 535000, vocab - 2000):
        part = g[:, v:v + 2000].t().contiguous() @ h.to(WIDE)
        size = g[:, v:v + 2000].t().abs().contiguous() @ h.to(WIDE).abs()
        inside(dw[v:v + 2000], part, size * (1.01 * U[torch.bfloat16] + 2 * bound) + part.abs() * 1.01 * U[torch.bfloat16], "dw")
    want = sum(g[:, v:v + 70000] @ w[v:v + 70000].to(WIDE) for v in range(0, vocab, 70000))
    assert (dh.to(WIDE) - want).norm() <= 2 * U[torch.bfloat16] * want.norm()


def test_linear_ce_against_differences(slz):
    h, w, labels, _ = ce_inputs(16, 32, 100, torch.float32, 70)
    labels[3] = IGNORED
    ones = torch.ones(16, device="cuda")
    _, lse = slz.linear_ce(h, w, labels)
    dh, dw = slz.linear_ce_grad(h, w, labels, lse, ones)
    step = 2.0 ** -6
    for grad, at, which in ((dh, h, 0), (dw, w, 1)):
        d = randn(tuple(at.shape), 71 + which)
        d /= d.norm()

        def total(x):
            return slz.linear_ce(x if which == 0 else h, w if which == 0 else x, labels)[0].to(WIDE).sum()

        diff = (total(at + step * d) - total(at - step * d)) / (2 * step)
        # losses to 2^-18 each; a third derivative of the loss along d is below the cube of what d moves the logits by
        moved = (d @ w.t()).abs().amax() if which == 0 else (h @ d.t()).abs().amax()
        assert abs(diff - (grad.to(WIDE) * d.to(WIDE)).sum()) < 16 * 2.0 ** -18 / step + 16 * moved.item() ** 3 * step ** 2


# ---- orthogonalised updates --------------------------------------------------------------------------------------------------------
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def orthogonalised(g, steps=5, coefficients=COEFFICIENTS, eps=1e-7):
    x = g.to(WIDE)
    if x.shape[0] > x.shape[1]:
        return orthogonalised(g.t(), steps, coefficients, eps).t()
    a, b, c = coefficients
    x = x / (x.norm() + eps)
    for _ in range(steps):
        s = x @ x.t().contiguous()
        x = a * x + (b * s + c * (s @ s)) @ x
    return x


def operand_error(g, bits, steps=5, coefficients=COEFFICIENTS, eps=1e-7):
    """What a result changes by when the operands of the three products of each step are rounded to `bits` bits (diagonals apart)."""
    x = g.to(WIDE)
    if x.shape[0] > x.shape[1]:
        x = x.t()

    def rounded(t):
        m, e = torch.frexp(t)
        return torch.ldexp(torch.round(m * 2.0 ** bits), e - bits)

    a, b, c = coefficients
    x = x / (x.norm() + eps)
    for _ in range(steps):
        o = rounded(x)
        s = o @ o.t().contiguous()
        d = torch.diag(s).clone()
        o2 = rounded(s - torch.diag(d))
        poly = b * (o2 + torch.diag(d)) + c * (o2 @ o2 + (d[:, None] + d[None, :]) * o2 + torch.diag(d * d))
        e = torch.diag(poly).clone()
        x = (a + e)[:, None] * x + rounded(poly - torch.diag(e)) @ o
    want = orthogonalised(g, steps, coefficients, eps)
    return ((x if g.shape[0] <= g.shape[1] else x.t()) - want).norm() / want.norm()


def check_update(slz, g, **kw):
    got = slz.orthogonalize(g, **kw)
    assert got.dtype == g.dtype and got.shape == g.shape
    bits, u = (11, U[torch.bfloat16]) if g.dtype == torch.bfloat16 else (22, U[g.dtype])
    for one, result in zip(g if g.dim() == 3 else g[None], got if g.dim() == 3 else got[None]):
        want = orthogonalised(one.cpu(), **kw)
        # four times what rounding the operands does (its pattern is another one), sums in 32 bits over min and max side grown by the steps, the result's type
        grown = max(one.shape) ** 0.5 * 2.0 ** -24 * COEFFICIENTS[0] ** kw.get("steps", 5)
        assert (result.cpu().to(WIDE) - want).norm() <= (4 * operand_error(one.cpu(), bits, **kw) + grown + u) * want.norm()
    return got


UPDATES = [(1, 1), (1, 9), (7, 1), (2, 3), (8, 8), (16, 100), (65, 33), (128, 784), (784, 128), (128, 128), (130, 131), (257, 300), (300, 256), (512, 512), (40, 2000),
           (128, 129), (100, 257), (33, 1100), (5000, 30), (64, 513), (3, 20000), (129, 3000), (2500, 200)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", UPDATES)
def test_orthogonalize_is_the_formula(slz, dtype, rows, cols):
    check_update(slz, randn((rows, cols), rows + cols, dtype, slack=(rows + cols) % 3, std=1e-3))


@pytest.mark.parametrize("dtype", TYPES)
def test_orthogonalize_batches_and_arguments(slz, dtype):
    g = randn((5, 48, 72), 1, dtype, slack=3)
    all_of = check_update(slz, g)
    for i in range(5):
        assert torch.equal(slz.orthogonalize(g[i]), all_of[i])
    assert torch.equal(slz.orthogonalize(g[::2]), all_of[::2])
    for rows, cols in ((100, 700), (20, 5000), (140, 2000)):         # slices and ranges of several matrices
        check_update(slz, randn((3, rows, cols), 3, dtype, slack=1))
    check_update(slz, g[0], steps=0)
    check_update(slz, g[0], steps=1)
    check_update(slz, g[1], steps=3, coefficients=(2.0, -1.5, 0.5))
    check_update(slz, g[1].t().contiguous(), steps=2, eps=0.5)
    assert slz.orthogonalize(g[:0]).shape == (0, 48, 72)
    assert slz.orthogonalize(g[0, :0]).shape == (0, 72)


@pytest.mark.parametrize("dtype", TYPES)
def test_orthogonalize_small_singular_values(slz, dtype):
    # singular values over three decades: the small ones grow by the first coefficient each step and must not drown in rounding
    u, _ = torch.linalg.qr(randn((96, 96), 2).to(WIDE).cpu())
    v, _ = torch.linalg.qr(randn((160, 96), 3).to(WIDE).cpu())
    g = (u @ torch.diag(torch.logspace(0, -3, 96, dtype=WIDE)) @ v.t()).to(dtype).cuda()
    check_update(slz, g)


def test_orthogonalize_special_values(slz):
    for dtype in TYPES:
        assert (slz.orthogonalize(torch.zeros((20, 30), dtype=dtype, device="cuda")) == 0).all()
    g = randn((20, 30), 4)
    g[3, 4] = float("nan")
    assert torch.isnan(slz.orthogonalize(g)).all()
    g = randn((20, 30), 5)
    for scale in (1e-30, 1e30):                       # squares leave 32 bits
        want = orthogonalised((g * scale).cpu(), eps=0.0)
        got = slz.orthogonalize(g * scale, eps=0.0).cpu().to(WIDE)
        assert (got - want).norm() <= 1e-3 * want.norm()
    g[3, 4] = float("inf")
    assert not torch.isfinite(slz.orthogonalize(g)).all()


# ---- all ----------------------------------------------------------------------------------------------------------------------------
def calls(slz):
    x = randn((70, 200), 1, torch.bfloat16)
    w, sw = int8((90, 200), 2), scales(90, 3)
    a, sa = int8((70, 200), 4), scales(70, 5)
    dy = randn((70, 90), 6, torch.float16)
    h, v, labels, dloss = ce_inputs(70, 64, 1000, torch.float16, 7)
    lse = slz.linear_ce(h, v, labels)[1]
    g = randn((2, 70, 90), 8, torch.bfloat16)
    one = randn((1, 2048), 9, torch.bfloat16)
    wide, s_wide = int8((700, 2048), 10), scales(700, 11)
    return [lambda: slz.quantize_i8(x), lambda: slz.linear_i8(x, w, sw), lambda: slz.matmul_i8(a, sa, w, sw), lambda: slz.matmul_i8_grad(dy, a, sa, w, sw),
            lambda: slz.linear_ce(h, v, labels), lambda: slz.linear_ce_grad(h, v, labels, lse, dloss), lambda: slz.orthogonalize(g),
            lambda: slz.linear_i8(one, wide, s_wide)]


def leaves(v):
    return list(v) if isinstance(v, tuple) else [v]


def test_the_same_inputs_give_the_same_bits_on_any_stream(slz):
    for call in calls(slz):
        first = [t.clone() for t in leaves(call())]
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            again = [leaves(call()) for _ in range(3)]
        s.synchronize()
        for got in again:
            for p, q in zip(first, got):
                assert torch.equal(p, q)


def test_calls_can_be_captured_and_replayed(slz):
    for call in calls(slz):
        want = [t.clone() for t in leaves(call())]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = leaves(call())
        for _ in range(4):
            for t in out:
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            for p, q in zip(want, out):
                assert torch.equal(p, q)
            call()


def test_the_binding_refuses(slz):
    x, w, s = randn((8, 32), 1), int8((4, 32), 2), scales(4, 3)
    h, v, labels, dloss = ce_inputs(8, 32, 50, torch.bfloat16, 4)
    with pytest.raises(TypeError):
        slz.linear_i8(x.double(), w, s)
    with pytest.raises(TypeError):
        slz.linear_i8(x, w.to(torch.int16), s)
    with pytest.raises(TypeError):
        slz.linear_i8(x, w, s.half())
    with pytest.raises(TypeError):
        slz.linear_ce(h, v, labels.int())
    with pytest.raises(TypeError):
        slz.linear_ce(h, v.float(), labels)
    with pytest.raises(TypeError):
        slz.matmul_i8(w, s, w, s, torch.int32)
    with pytest.raises(ValueError):
        slz.linear_i8(x[:, :31], w, s)
    with pytest.raises(ValueError):
        slz.linear_i8(x, w, s[:3])
    with pytest.raises(ValueError):
        slz.linear_i8(x.t(), w[:, :8], s)              # no unit stride along the rows
    with pytest.raises(ValueError):
        slz.linear_i8(x[0].expand(4, 32), w, s)        # rows overlap
    with pytest.raises(ValueError):
        slz.linear_ce(h, v, labels[:5])
    with pytest.raises(ValueError):
        slz.linear_ce_grad(h, v, labels, dloss[:5], dloss)
    with pytest.raises(ValueError):
        slz.matmul_i8_grad(x, w, s, w, s)
    with pytest.raises(ValueError):
        slz.orthogonalize(x, steps=65)
    with pytest.raises(ValueError):
        slz.orthogonalize(x[0])
    with pytest.raises(slz.SlzError):
        slz.linear_ce(h, v[:0], labels)


def test_the_example_learns_and_answers_in_8_bits():
    import examples.clear_step as example
    losses, right, one, among = example.train(steps=40)
    # ten classes: the loss begins near log 10 and the classes are far apart (0.3 sqrt(784) = 8 deviations)
    assert losses[0] > 1.5 and sum(losses[-5:]) / 5 < 0.5 * losses[0]
    assert right > 0.9
    assert torch.equal(one, among)                     # an input answered alone and among others
