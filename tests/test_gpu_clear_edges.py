"""Edges of the operators of include/silenzio_clear.h: values that must have no influence, numbers far apart, lengths beyond a launch's."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_clear import COEFFICIENTS, IGNORED, LEAST, TYPES, U, WIDE, ce_inputs, inside, int8, orthogonalised, quantised, randn, scales, slz  # noqa: E402,F401


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("inner,vocab", [(64, 300), (128, 10)])
def test_dloss_of_tokens_that_do_not_count_changes_nothing(slz, dtype, inner, vocab):  # noqa: F811
    h, w, labels, dloss = ce_inputs(40, inner, vocab, dtype, 42)
    dloss *= 1e-3
    labels[7] = labels[30] = IGNORED
    lse = slz.linear_ce(h, w, labels)[1]
    want = slz.linear_ce_grad(h, w, labels, lse, dloss)
    assert all((t != 0).any() for t in want)
    for large in (1.0, 1e12, -3e38):
        dloss[7], dloss[30] = large, -large
        for got, t in zip(slz.linear_ce_grad(h, w, labels, lse, dloss), want):
            assert torch.equal(got, t)
    # a label outside the vocabulary makes its own row NaN, and dw; the other tokens' rows stay what they are
    labels[7] = vocab
    dh, _ = slz.linear_ce_grad(h, w, labels, lse, dloss)
    rest = [t for t in range(40) if t != 7]
    assert torch.isnan(dh[7]).all() and torch.equal(dh[rest], want[0][rest])


@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_of_rows_with_small_scales(slz, dtype):  # noqa: F811
    # one term a sum, so that each value of scale x integer shows by itself; scales from 1 down to 2^-21
    n, k = 64, 96
    a, b = int8((n, k), 1), int8((n, k), 2)
    s = 1.37 * 2.0 ** (-torch.arange(n, device="cuda") / 3)
    dy = torch.zeros(n, n, device="cuda", dtype=dtype)
    dy.fill_diagonal_(200.0)
    want_a, want_b = 200 * b.to(WIDE) * s.to(WIDE)[:, None], 200 * a.to(WIDE) * s.to(WIDE)[:, None]
    for got, want in zip(slz.matmul_i8_grad(dy, a, s, b, s), (want_a, want_b)):
        # the value to the type (f32: 24 bits), the products in 32 bits, the result to the type
        value = U[dtype] if dtype != torch.float32 else 2.0 ** -21
        inside(got, want, want.abs() * 1.01 * (value + U[dtype] + 8 * 2.0 ** -24) + LEAST[dtype], "gradient")


def updates(rows, cols):
    """Gradients with entries far apart: a few strong directions, every other row a thousandth of the rest."""
    g = randn((rows, cols), rows + cols)
    yield g + 30 * randn((rows, 4), 1) @ randn((4, cols), 2)
    g[::2] *= 1e-3
    yield g


@pytest.mark.parametrize("rows,cols", [(64, 512), (128, 8000), (8000, 128), (200, 300), (2000, 2100), (2100, 2000)])
def test_updates_keep_small_entries(slz, rows, cols):  # noqa: F811
    # coefficients (1, 0, 0) only hold X: 22 bits or 2^-35 each time, and some roundings in 32 bits
    for g in updates(rows, cols):
        want = orthogonalised(g, steps=0)
        for steps in (0, 1, 3):
            got = slz.orthogonalize(g, steps=steps, coefficients=(1.0, 0.0, 0.0))
            inside(got, want, max(steps, 1) * (want.abs() * (2.0 ** -22 + 4 * 2.0 ** -24) + 2.0 ** -35), "%d steps" % steps)


@pytest.mark.parametrize("rows,cols", [(128, 8000), (300, 3000)])
def test_updates_are_as_good_as_in_32_bits(slz, rows, cols):  # noqa: F811
    a, b, c = COEFFICIENTS
    for g in updates(rows, cols):
        want = orthogonalised(g)
        x = g / g.norm()
        for _ in range(5):
            s = x @ x.t().contiguous()
            x = a * x + (b * s + c * (s @ s)) @ x
        # numbers of 22 bits in place of 24
        assert (slz.orthogonalize(g).to(WIDE) - want).norm() <= 4 * (x.to(WIDE) - want).norm()


def test_quantize_of_more_rows_than_a_launch_takes(slz):  # noqa: F811
    # a workgroup of 256 a row: 2^24 rows are 2^32 threads
    rows = 2 ** 24 + 3
    x = randn((rows, 1), 1, torch.bfloat16)
    q, scale = slz.quantize_i8(x)
    want_q, want_scale = quantised(x)
    assert np.array_equal(q.cpu().numpy(), want_q) and np.array_equal(scale.cpu().numpy(), want_scale)
    x = randn((rows, 16), 2, torch.bfloat16)
    w, sw = int8((3, 16), 3), scales(3, 4)
    y = slz.linear_i8(x, w, sw)
    for part in (slice(0, 1000), slice(2 ** 24 - 1000, rows)):
        assert torch.equal(y[part], slz.linear_i8(x[part].contiguous(), w, sw))


def test_product_of_more_tiles_than_a_launch_takes(slz):  # noqa: F811
    # tiles of 64 rows, workgroups of 256: 2^30 rows are 2^32 threads
    m, k = 2 ** 30 + 65, 16
    a = torch.randint(-128, 128, (m, k), device="cuda", dtype=torch.int8)
    b, sa, sb = int8((1, k), 2), torch.ones(m, device="cuda"), torch.ones(1, device="cuda")
    y = slz.matmul_i8(a, sa, b, sb, torch.float32)
    for first in range(0, m, 2 ** 25):
        part = slice(first, min(m, first + 2 ** 25))
        assert torch.equal(y[part, 0], (a[part].float() * b.float()).sum(1))          # whole numbers below 2^24


def test_loss_of_more_tokens_than_a_launch_takes(slz):  # noqa: F811
    # the join has 1024 threads for 16 tokens: 2^26 tokens are 2^32
    tokens, inner, vocab = 2 ** 26 + 21, 8, 17
    h, w = randn((tokens, inner), 1, torch.bfloat16), randn((vocab, inner), 2, torch.bfloat16)
    labels = torch.randint(0, vocab, (tokens,), device="cuda")
    loss, lse = slz.linear_ce(h, w, labels)
    for first in (0, 2 ** 25 + 5, 2 ** 26 - 2 ** 20):
        part = slice(first, min(tokens, first + 2 ** 21))
        one, two = slz.linear_ce(h[part].contiguous(), w, labels[part].contiguous())
        assert torch.equal(one, loss[part]) and torch.equal(two, lse[part])
        want = torch.logsumexp(h[part].to(WIDE) @ w.to(WIDE).t().contiguous(), 1)
        inside(lse[part], want, 2.0 ** -17, "lse")     # z of some ten, eight terms in 32 bits


def test_the_binding_refuses_lengths_beyond_32_bits(slz):  # noqa: F811
    # matrices without elements take no memory; 2^32 + 3 is not 3
    long = 2 ** 32 + 3
    tall, wide, three = torch.empty((long, 0), device="cuda"), torch.empty((0, long), device="cuda"), torch.empty((3, 0), device="cuda")
    labels, one = torch.empty(0, dtype=torch.int64, device="cuda"), scales(3, 1)
    for call in (lambda: slz.quantize_i8(wide), lambda: slz.linear_i8(tall, three.to(torch.int8)[:0], one[:0]), lambda: slz.linear_ce(wide, wide, labels),
                 lambda: slz.matmul_i8(wide.to(torch.int8), one[:0], wide.to(torch.int8), one[:0]),
                 lambda: slz.orthogonalize(tall), lambda: slz.orthogonalize(torch.empty((long, 0, 4), device="cuda"))):
        with pytest.raises(slz.SlzError):
            call()


def test_a_backward_pass_does_not_skip_what_autograd_cannot_do(slz):  # noqa: F811
    h, w, labels, dloss = ce_inputs(8, 32, 50, torch.float32, 4)
    b, s = int8((4, 32), 2), scales(4, 3)
    q, sq = slz.quantize_i8(h)
    lse = slz.linear_ce(h, w, labels)[1]
    plain = slz.linear_ce(h, w, labels)[0]
    assert not plain.requires_grad
    p = h.clone().requires_grad_()
    for result in (lambda: slz.linear_ce(p, w, labels)[0], lambda: slz.linear_i8(p, b, s), lambda: slz.orthogonalize(p), lambda: slz.quantize_i8(p)[1],
                   lambda: slz.linear_ce_grad(p, w, labels, lse, dloss)[1], lambda: slz.matmul_i8_grad(p[:, :4], q, sq, b, s, need_b=False)[0],
                   lambda: slz.matmul_i8(q, p[:, 0].contiguous(), b, s, torch.float32)):
        with pytest.raises(RuntimeError, match="autograd"):
            (result().sum() + p.sum()).backward()
        with torch.no_grad():
            assert not result().requires_grad
    assert torch.equal(slz.linear_ce(p, w, labels)[0].detach(), plain)
    assert not slz.quantize_i8(p)[0].requires_grad


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("weight", [(1 + 2.0 ** -8) / 32, (1 + 2.0 ** -11) / 32, 1 / 3584, 1 / 7])
def test_a_common_dloss_is_not_rounded(slz, dtype, weight):  # noqa: F811
    # all tokens alike: the rounding of dloss to the type would be one error of all of the gradient
    h, w, labels, dloss = ce_inputs(200, 128, 3000, dtype, 70)
    labels[::9] = IGNORED
    dloss[:] = weight
    lse = slz.linear_ce(h, w, labels)[1]
    g = torch.softmax(h.to(WIDE) @ w.to(WIDE).t().contiguous(), 1)
    counts = labels != IGNORED
    g[counts, labels[counts]] -= 1
    g *= torch.where(counts, dloss.to(WIDE), 0.0)[:, None]
    for got, want in zip(slz.linear_ce_grad(h, w, labels, lse, dloss), (g @ w.to(WIDE), g.t().contiguous() @ h.to(WIDE))):
        # root mean squares: -1 + p is off by 0.29 U (half a place below 1 at most), the result by 0.43 U, p by 0.43 U of its share of g, below a half:
        # together less than one and a half times the result's own
        own = (want.to(dtype).to(WIDE) - want).norm() if dtype != torch.float32 else 2.0 ** -20 * want.norm()
        assert (got.to(WIDE) - want).norm() <= 1.5 * own


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [(1 + 2.0 ** -8) / 64, (1 + 2.0 ** -11) / 64, 0.0123, 0.0, float("nan")])
def test_gradients_of_one_row(slz, dtype, scale):  # noqa: F811
    # one token: integers times one scale, each gradient of it rounded once
    n, k = 70, 300
    a, b = int8((1, k), 1), int8((n, k), 2)
    s, one, dy = torch.full((1,), scale, device="cuda"), scales(n, 3), randn((1, n), 4, dtype)
    _, db = slz.matmul_i8_grad(dy, a, s, b, one, need_a=False)
    want = dy.to(WIDE).t().contiguous() @ (a.to(WIDE) * s.to(WIDE))
    inside(db, want, (want.abs() * (1.01 * U[dtype] + 3 * 2.0 ** -24)).nan_to_num() + LEAST[dtype], "db")
    da, _ = slz.matmul_i8_grad(dy.t().contiguous(), b, one, a, s, need_b=False)
    inside(da, want, (want.abs() * (1.01 * U[dtype] + 3 * 2.0 ** -24)).nan_to_num() + LEAST[dtype], "da")
