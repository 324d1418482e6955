"""Edges of the operators of include/silenzio_clear.h: values that must have no influence, numbers far apart, lengths beyond a launch's."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_clear import IGNORED, LEAST, TYPES, U, WIDE, ce_inputs, inside, int8, slz  # noqa: E402,F401


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
