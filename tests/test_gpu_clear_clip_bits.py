"""Clipping with a factor of 1 leaves the elements' bits, infinities' and those of any NaN, wherever they lie."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_clear import TYPES, slz  # noqa: E402,F401


@pytest.mark.parametrize("dtype", TYPES)
def test_elements_below_the_limit_keep_their_bits(slz, dtype):  # noqa: F811
    whole = torch.int32 if dtype == torch.float32 else torch.int16
    if dtype == torch.float32:
        # NaN of any payload, quiet and not, zeros, subnormals, infinities, and anything
        gen = torch.Generator(device="cuda").manual_seed(1)
        bits = torch.randint(-(1 << 31), 1 << 31, (1 << 16,), device="cuda", generator=gen, dtype=torch.int64)
        bits[::4] = bits[::4] & ~0x7f800000 | 0x7f800000
        bits[1::4] &= ~0x7f800000
        bits[:4] = torch.tensor([0x7f800001, -0x7fffff, 0x7f800000, 1], device="cuda")
        bits = bits.to(whole)
    else:
        bits = torch.arange(-(1 << 15), 1 << 15, device="cuda").to(whole)          # all of them
    for rows, cols in ((1, 1 << 16), (1 << 13, 8), (1 << 14, 3), (9, 7001), (1 << 16, 1)):
        for slack_g, slack_o in ((0, 0), (1, 0), (0, 1), (3, 2)):
            count = rows * cols
            g = torch.zeros((rows, cols + slack_g), dtype=whole, device="cuda")
            g[:, :cols] = bits[:count].view(rows, cols)
            out = torch.full((rows, cols + slack_o), 5, dtype=whole, device="cuda")
            given = torch.tensor(0.5, device="cuda")
            slz.clip_by_norm([g.view(dtype)[:, :cols]], 1.0, norm=given, out=[out.view(dtype)[:, :cols]])
            assert torch.equal(out[:, :cols], g[:, :cols]) and (out[:, cols:] == 5).all()
    # tensors of a few elements, from odd places on
    g, out = bits.clone(), torch.zeros_like(bits)
    at = [(i * 31, i * 31 + 1 + i % 29) for i in range(1000)]
    slz.clip_by_norm([g.view(dtype)[a:b] for a, b in at], 1.0, norm=given, out=[out.view(dtype)[a:b] for a, b in at])
    assert all(torch.equal(out[a:b], g[a:b]) for a, b in at)
