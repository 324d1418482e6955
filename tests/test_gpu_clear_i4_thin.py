"""One and two rows by many rows of 4-bit weights, on both sides of where a workgroup has more of them (f32, 12288), against the formula in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_clear import TYPES, WIDE, inside, randn, slz  # noqa: E402,F401
from tests.test_gpu_clear_i4 import bounds, unpack, values  # noqa: E402


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [8192, 8193, 12288, 12289, 12305, 16383, 16384])
def test_few_rows_by_many(slz, dtype, n):  # noqa: F811
    for m, k, group in ((1, 1, 32), (1, 260, 64), (2, 1025, 128), (2, 640, 32)):
        gen = torch.Generator(device="cuda").manual_seed(n + m)
        q = torch.randint(0, 256, (n, (k + 127) // 128 * 64), dtype=torch.uint8, device="cuda", generator=gen)
        scale = torch.rand((n, (k + group - 1) // group), device="cuda", generator=gen) + 0.01
        w = values(unpack(q, k), scale, group)
        x = randn((m, k), k, dtype, slack=1)
        want = x.to(WIDE) @ w.t()
        inside(slz.linear_i4(x, q, scale, group), want, bounds(x.to(WIDE), w, want, dtype, k, rounded=False), "y")
