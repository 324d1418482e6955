"""Products with 4-bit weights whose values are laid out in the type first (tests/clear_i4_laid_out.py): what they round, what they keep of infinities, NaN, small and far-apart numbers, and
that they repeat themselves on any stream and in a captured graph."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.clear_i4_laid_out import SHAPES  # noqa: E402
from tests.test_gpu_clear import LEAST, TYPES, U, WIDE, inside, randn, slz  # noqa: E402,F401
from tests.test_gpu_clear_i4 import bounds, unpack, values  # noqa: E402


def codes(n, k, seed):
    """Any 4-bit rows, the places past the rows' ends among them, and zeros with a sign."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, 256, (n, (k + 127) // 128 * 64), dtype=torch.uint8, device="cuda", generator=gen)


def held(q, scale, group, cols, dtype):
    """The values as the type holds them, in 64 bits: scale times entry in 32 bits, f16 of it times 2^12 and divided by the power of two above the largest scale."""
    v = torch.from_numpy(unpack(q, cols)).cuda().float() * scale.repeat_interleave(group, 1)[:, :cols]
    if dtype == torch.float32:
        return v.to(WIDE)
    if dtype == torch.bfloat16:
        return v.to(dtype).to(WIDE)
    by = 2.0 ** (12 - torch.frexp(scale.abs().amax())[1].item())
    return (v * by).to(dtype).to(WIDE) / by


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_nothing_is_rounded_but_the_values(slz, dtype, m, n, k):  # noqa: F811
    # with the values as the type holds them, the sums have 32 bits and are rounded once: no term of an operand's rounding is left in the bound for 16-bit types
    for group, decades in ((32, 1), (64, 4), (128, 13)):                           # 13: f16 has no number for most of the values
        q = codes(n, k, m + group)
        gen = torch.Generator(device="cuda").manual_seed(group)
        scale = 10.0 ** (-decades * torch.rand((n, (k + group - 1) // group), device="cuda", generator=gen))
        x = randn((m, k), k, dtype, slack=group % 3)
        w = held(q, scale, group, k, dtype)
        want = x.to(WIDE) @ w.t()
        y = slz.linear_i4(x, q, scale, group)
        inside(y, want, bounds(x.to(WIDE), w, want, dtype, k, rounded=False), "y, group %d" % group)
        for _ in range(3):
            assert torch.equal(y, slz.linear_i4(x, q, scale, group))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_infinities_and_nan_stay_where_they_belong(slz, dtype, m, n, k):  # noqa: F811
    group = 64
    q = codes(n, k, 3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    scale = torch.rand((n, (k + group - 1) // group), device="cuda", generator=gen) + 0.01
    x = randn((m, k), 5, dtype, slack=3)
    x.as_strided((m - 1, 3), (k + 3, 1), k).fill_(float("nan"))                    # between the rows
    want = slz.linear_i4(x.contiguous(), q, scale, group)
    assert torch.isfinite(want).all() and torch.equal(slz.linear_i4(x, q, scale, group), want)
    # a NaN scale is its column's, and has no part in what f16's values are relative to
    bad = scale.clone()
    bad[9, 0] = float("nan")
    rest = [i for i in range(n) if i != 9]
    top = scale.argmax().item() // scale.shape[1]
    assert top != 9
    got = slz.linear_i4(x, q, bad, group)
    assert torch.isnan(got[:, 9]).all() and torch.equal(got[:, rest], want[:, rest])
    # an infinity or NaN in x is its row's
    for value in (float("inf"), float("-inf"), float("nan")):
        y = x.clone()
        y[m // 2, k // 2] = value
        others = [i for i in range(m) if i != m // 2]
        got = slz.linear_i4(y, q, scale, group)
        assert not torch.isfinite(got[m // 2]).any() and torch.equal(got[others], want[others])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_values_of_any_scale(slz, dtype, m, n, k):  # noqa: F811
    # one term a sum, so that each value shows by itself; scales from 1 down to 2^-24, and all of them far from 1
    group = 32
    q = codes(n, k, 6)
    at = torch.arange(m, device="cuda") * 5 % k
    for far in (1.0, 2.0 ** -60, 2.0 ** 40):
        s = (far * 1.37 * 2.0 ** (-(torch.arange(n, device="cuda", dtype=WIDE) % 73) / 3)).float()[:, None].expand(n, (k + group - 1) // group).contiguous()
        w = values(unpack(q, k), s, group)
        x = torch.zeros((m, k), device="cuda", dtype=dtype)
        x[torch.arange(m, device="cuda"), at] = 200.0
        want = 200 * w.t()[at]
        fits = want.abs() < 0.99 * torch.finfo(dtype).max
        value = U[dtype] if dtype != torch.float32 else 2.0 ** -21
        bound = want.abs() * 1.01 * (value + U[dtype] + 8 * 2.0 ** -24) + LEAST[dtype]
        y = slz.linear_i4(x, q, s, group)
        inside(torch.where(fits, y, 0), torch.where(fits, want, 0), bound, "scales of %g" % far)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_small_inputs_are_not_lost(slz, dtype, m, n, k):  # noqa: F811
    # inputs below the type's smallest ordinary number, times scales that bring the results back
    group = 128
    q = codes(n, k, 7)
    scale = torch.full((n, (k + group - 1) // group), 2.0 ** 13 if dtype == torch.float16 else 2.0 ** 120, device="cuda")
    w = values(unpack(q, k), scale, group)
    step = 2.0 ** -24 if dtype == torch.float16 else 2.0 ** -133
    x = (torch.randint(-60, 61, (m, k), device="cuda", generator=torch.Generator(device="cuda").manual_seed(m)).to(WIDE) * step).to(dtype)
    assert (x != 0).any() and x.abs().max() < torch.finfo(dtype).tiny
    want = x.to(WIDE) @ w.t()
    inside(slz.linear_i4(x, q, scale, group), want, bounds(x.to(WIDE), w, want, dtype, k), "y")


def test_the_same_bits_on_two_streams_at_once_and_replayed(slz):  # noqa: F811
    for dtype in TYPES:
        for m, n, k in SHAPES:
            sides = []
            for seed in (1, 2):
                gen = torch.Generator(device="cuda").manual_seed(seed)
                # scales of other sizes on each side: f16's units differ
                sides.append((randn((m, k), seed, dtype, slack=1), codes(n, k, seed), (torch.rand((n, (k + 63) // 64), device="cuda", generator=gen) + 0.01) * 1000.0 ** (seed - 1)))
            want = [slz.linear_i4(*s, 64).clone() for s in sides]
            torch.cuda.synchronize()
            streams, got = (torch.cuda.Stream(), torch.cuda.Stream()), []
            for _ in range(3):
                for i, stream in enumerate(streams):
                    with torch.cuda.stream(stream):
                        got.append((i, slz.linear_i4(*sides[i], 64)))
            torch.cuda.synchronize()
            for i, y in got:
                assert torch.equal(y, want[i])
            graphs, out = [], []
            for s in sides:
                graphs.append(torch.cuda.CUDAGraph())
                with torch.cuda.graph(graphs[-1]):
                    out.append(slz.linear_i4(*s, 64))
            for _ in range(4):
                for y in out:
                    y.zero_()
                for graph in graphs:
                    graph.replay()
                assert torch.equal(slz.linear_i4(*sides[0], 64), want[0])
                torch.cuda.synchronize()
                assert all(torch.equal(y, t) for y, t in zip(out, want))
