"""Every tiling of the tiled matrix product of include/silenzio_clear.h against the formulas in 64 bits (shapes: tests/clear_tilings.py)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests import clear_tilings  # noqa: E402
from tests.test_gpu_clear import COEFFICIENTS, IGNORED, LEAST, U, WIDE, ce_inputs, check_ce, inside, int8, operand_error, orthogonalised, randn, scales, slz  # noqa: E402,F401

HALVES = (torch.bfloat16, torch.float16)


def each(table, flag):
    """(shape, type) of every row, once for each type that takes its tilings."""
    return [(row[0], t) for row in table for t in flag(row)]


@pytest.mark.parametrize("shape", [row[0] for row in clear_tilings.PRODUCTS])
def test_products(slz, shape):  # noqa: F811
    m, n, k = shape
    a, b = int8((m, k), 1, k % 3), int8((n, k), 2)
    sa, sb = scales(m, 3), scales(n, 4)
    y = slz.matmul_i8(a, sa, b, sb, torch.bfloat16)
    want = (a.to(WIDE) @ b.to(WIDE).t()) * sa.to(WIDE)[:, None] * sb.to(WIDE)[None, :]
    # the sum to 32 bits, the scales' product, their product, and the type's own rounding
    inside(y, want, want.abs() * (3.01 * 2.0 ** -24 + 1.01 * U[torch.bfloat16]) + LEAST[torch.bfloat16], "y")


@pytest.mark.parametrize("shape,dtype", each(clear_tilings.GRADS, lambda row: (torch.float32,) if row[1] else HALVES))
def test_gradients_of_products(slz, shape, dtype):  # noqa: F811
    m, n, k = shape
    dy = randn((m, n), 8, dtype, slack=k % 3)
    a, b = int8((m, k), 9, slack=m % 2), int8((n, k), 10)
    sa, sb = scales(m, 11), scales(n, 12)
    da, db = slz.matmul_i8_grad(dy, a, sa, b, sb)
    A, B, D = a.to(WIDE) * sa.to(WIDE)[:, None], b.to(WIDE) * sb.to(WIDE)[:, None], dy.to(WIDE)
    turned = D.t().contiguous()
    for got, want, size, terms, largest, what in ((da, D @ B, D.abs() @ B.abs(), n, sb.max(), "da"), (db, turned @ A, turned.abs() @ A.abs(), m, sa.max(), "db")):
        # values rounded to the type (f32: in three pieces), sums, result; f16 values below 2^-14 of the largest scale lose bits
        bound = size * ((1.01 * U[dtype] if dtype != torch.float32 else 2.0 ** -21) + (terms + 4) * 2.0 ** -24) + want.abs() * 1.01 * U[dtype] + LEAST[dtype]
        if dtype == torch.float16:
            bound = bound + 2.0 ** -24 * largest.item() * 2 * terms * D.abs().max()
        inside(got, want, bound, what)


@pytest.mark.parametrize("shape,dtype", each(clear_tilings.LOSSES, lambda row: (torch.float32,) if row[1] else HALVES))
def test_losses_and_their_gradients(slz, shape, dtype):  # noqa: F811
    tokens, inner, vocab = shape
    h, w, labels, dloss = ce_inputs(tokens, inner, vocab, dtype, 20, slack=(tokens + vocab) % 3)
    labels[::7] = vocab - 1
    labels[3::5] = IGNORED
    check_ce(slz, h, w, labels, dloss)


@pytest.mark.parametrize("shape,dtype", each(clear_tilings.UPDATES, lambda row: (torch.float32, torch.float16) if row[1] else (torch.bfloat16,)))
def test_updates(slz, shape, dtype):  # noqa: F811
    batch, m, n = shape
    g = randn((batch, m, n), m + n, dtype, slack=n % 3, std=1e-3)
    got = slz.orthogonalize(g)
    bits, steps = 11 if dtype == torch.bfloat16 else 22, 5
    for one, result in zip(g, got):
        want = orthogonalised(one)
        # four times what rounding the operands does (its pattern is another one), sums in 32 bits grown by the steps, the result's type
        near = 4 * operand_error(one, bits) + n ** 0.5 * 2.0 ** -24 * COEFFICIENTS[0] ** steps + U[dtype]
        off = result.to(WIDE) - want
        assert off.norm() <= near * want.norm()
        # and no part of it far off: blocks of 64 x 64 have their share of the error, within a factor of 8
        for r in range(0, m, 64):
            for c in range(0, n, 64):
                part = off[r:r + 64, c:c + 64]
                assert part.norm() <= 8 * near * want.norm() * (part.numel() / want.numel()) ** 0.5, (r, c)
    if batch > 1:                                      # taller than wide: the transposed result
        turned = slz.orthogonalize(g.transpose(1, 2).contiguous())
        assert torch.equal(turned, got.transpose(1, 2).contiguous())
