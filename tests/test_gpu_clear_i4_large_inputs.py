"""Products with 4-bit weights of inputs up to the largest numbers of their type: what a group sums up to before its scale brings it down leaves 32 bits by itself, the result does not.
Only the kernels that stream the weights sum groups (tests/clear_i4_routes.py has shapes of each)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.clear_i4_routes import ROUTES  # noqa: E402
from tests.test_gpu_clear import WIDE, inside, randn, slz  # noqa: E402,F401
from tests.test_gpu_clear_i4 import bounds, unpack, values  # noqa: E402

STREAMED = [(shape, dtype) for shape, wide, (way, _) in ROUTES if way != "tiles" and shape[1] * shape[2] < 1 << 24 for dtype in ((torch.float32,) if wide else (torch.bfloat16, torch.float16))]
NAMES = ["%s-%s" % ("x".join(map(str, s)), str(d)[6:]) for s, d in STREAMED]


def codes(n, k, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, 256, (n, (k + 127) // 128 * 64), dtype=torch.uint8, device="cuda", generator=gen)


@pytest.mark.parametrize("shape,dtype", STREAMED, ids=NAMES)
def test_groups_do_not_overflow(slz, shape, dtype):  # noqa: F811
    m, n, k, group = shape
    gen = torch.Generator(device="cuda").manual_seed(k)
    x = ((torch.rand((m, k), device="cuda", generator=gen) * 2 - 1) * (0.99 * torch.finfo(dtype).max)).to(dtype)
    x[:, ::2] = x[:, ::2].abs()
    q = codes(n, k, m)
    q[0] = 0x77                                        # all entries 7
    # at most 20001 terms of 7 max: below max / 2
    scale = (torch.rand((n, (k + group - 1) // group), device="cuda", generator=gen) + 1.0) * 2.0 ** -20
    w = values(unpack(q, k), scale, group)
    want = x.to(WIDE) @ w.t()
    assert want.abs().max() < torch.finfo(dtype).max / 2
    inside(slz.linear_i4(x, q, scale, group), want, bounds(x.to(WIDE), w, want, dtype, k, rounded=False), "y")


@pytest.mark.parametrize("shape,dtype", [s for s in STREAMED if s[1] != torch.float16], ids=[i for i in NAMES if "float16" not in i.replace("bfloat16", "")])
def test_groups_with_small_and_large_scales_side_by_side(slz, shape, dtype):  # noqa: F811
    m, n, k, group = shape
    gen = torch.Generator(device="cuda").manual_seed(k + 1)
    q = codes(n, k, m + 1)
    power = torch.randint(0, 6, (n, (k + group - 1) // group), device="cuda", generator=gen)
    scale = torch.tensor([2.0 ** 100, 1.5 * 2.0 ** 99, 2.0 ** 101, 1.0, -(2.0 ** 100), 2.0 ** 90], device="cuda")[power]
    w = values(unpack(q, k), scale, group)
    # ordinary inputs, and inputs below the smallest ordinary number
    small = (torch.randint(-60, 61, (m, k), device="cuda", generator=gen).to(WIDE) * 2.0 ** -133).to(dtype)
    assert small.abs().max() < torch.finfo(dtype).tiny
    for x in (randn((m, k), 2, dtype), small):
        want = x.to(WIDE) @ w.t()
        inside(slz.linear_i4(x, q, scale, group), want, bounds(x.to(WIDE), w, want, dtype, k, rounded=False), "y")
