"""Products with 4-bit weights at shapes that take each of their kernels (tests/clear_i4_routes.py), against the formula in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.clear_i4_routes import ROUTES  # noqa: E402
from tests.test_gpu_clear import WIDE, inside, randn, slz  # noqa: E402,F401
from tests.test_gpu_clear_i4 import bounds, unpack, values  # noqa: E402


@pytest.mark.parametrize("shape,wide,taken", ROUTES, ids=["%s-%s" % ("x".join(map(str, s)), "f32" if w else "16") for s, w, _ in ROUTES])
def test_products(slz, shape, wide, taken):  # noqa: F811
    m, n, k, group = shape
    gen = torch.Generator(device="cuda").manual_seed(m + n)
    # any codes, the places past the rows' ends among them, and zeros with a sign
    q = torch.randint(0, 256, (n, (k + 127) // 128 * 64), dtype=torch.uint8, device="cuda", generator=gen)
    scale = torch.rand((n, (k + group - 1) // group), device="cuda", generator=gen) + 0.01
    w = values(unpack(q, k), scale, group)
    for dtype in (torch.float32,) if wide else (torch.bfloat16, torch.float16):
        for slack in (0, 3):
            x = randn((m, k), k, dtype, slack=slack, skip=slack)
            y = slz.linear_i4(x, q, scale, group)
            want = x.to(WIDE) @ w.t()
            # no value is rounded on the way that streams them
            inside(y, want, bounds(x.to(WIDE), w, want, dtype, k, rounded=taken[0] == "tiles"), "y")
            assert torch.equal(y, slz.linear_i4(x, q, scale, group))
