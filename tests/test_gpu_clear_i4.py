"""Layers with 4-bit weights (include/silenzio_clear.h) against their formulas in 64 bits.

U is a type's unit roundoff.  A sum of n products in 32 bits is off by at most (n + 2) 2^-24 of the sum of their magnitudes; an operand rounded to a type
adds U of it; three bf16 carry a 32-bit number, and the products of them that are left out are below 2^-21 of the magnitudes."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_clear import LEAST, TYPES, U, WIDE, inside, leaves, randn, slz  # noqa: E402,F401

GROUPS = (32, 64, 128)


def pack(q):
    """Whole numbers from -7 to 7, int [rows][cols] on the host, to 4-bit rows by the header's definition."""
    q = np.asarray(q)
    rows, cols = q.shape
    out = np.zeros((rows, (cols + 127) // 128 * 64), dtype=np.uint8)
    k = np.arange(cols)
    block, s, j, e = k // 128, k % 128 // 32, k % 32 // 8, k % 8
    at, shift = block * 64 + (4 * j + s) * 4 + e % 4, 4 * (e // 4)
    for c in range(cols):
        out[:, at[c]] |= ((np.abs(q[:, c]) | (q[:, c] < 0) * 8) << shift[c]).astype(np.uint8)
    return out


def unpack(packed, cols):
    packed = packed.cpu().numpy()
    k = np.arange(cols)
    block, s, j, e = k // 128, k % 128 // 32, k % 32 // 8, k % 8
    code = packed[:, block * 64 + (4 * j + s) * 4 + e % 4] >> (4 * (e // 4)) & 15
    return np.where(code & 8, -1, 1) * (code & 7).astype(np.int64)


def weights(n, k, group, seed, dead=True):
    """(integers, 4-bit rows, scales): scales over three decades, one row of zeros."""
    rng = np.random.default_rng(seed)
    q = rng.integers(-7, 8, (n, k))
    groups = (k + group - 1) // group
    scale = (10.0 ** rng.uniform(-4, -1, (n, groups))).astype(np.float32)
    if dead and n > 2:
        scale[1] = 0
    return q, torch.from_numpy(pack(q)).cuda(), torch.from_numpy(scale).cuda()


def values(q, scale, group):
    """The values in 64 bits, on the card."""
    q = torch.from_numpy(np.asarray(q)).cuda().to(WIDE)
    return q * scale.to(WIDE).repeat_interleave(group, 1)[:, :q.shape[1]]


# ---- quantisation -------------------------------------------------------------------------------------------------------------------
def quantised(w, group):
    """The definition.  7 w / top is a quotient of whole numbers of up to 27 and 24 bits (w and top scaled): it is a half exactly, or at least 2^-28 from one, so its
    rounding to 53 bits moves it neither onto a half nor across one."""
    w = w.to(WIDE).cpu().numpy()
    rows, cols = w.shape
    q, scale = np.zeros((rows, cols), dtype=np.int64), np.zeros((rows, (cols + group - 1) // group), dtype=np.float32)
    for i in range(scale.shape[1]):
        part = w[:, i * group:(i + 1) * group]
        top = np.abs(part).max(axis=1)
        with np.errstate(all="ignore"):
            n = np.rint(7 * part / top[:, None])
            q[:, i * group:(i + 1) * group] = np.where((top > 0) & np.isfinite(top), 1, 0)[:, None] * np.nan_to_num(n, posinf=0, neginf=0)
            scale[:, i] = np.where(np.isfinite(top), top.astype(np.float32) / np.float32(7), np.float32("nan"))
    return q, scale


@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,slack", [(1, 1, 0), (3, 7, 2), (2, 31, 0), (5, 33, 1), (4, 128, 0), (7, 129, 3), (128, 784, 0), (2, 1000, 1), (33, 4096, 8), (3, 20001, 0), (40000, 5, 0)])
def test_quantize_is_the_definition(slz, dtype, group, rows, cols, slack):  # noqa: F811
    w = randn((rows, cols), rows + cols, dtype, slack)
    w[rows // 2] *= 1e-3
    q, scale = slz.quantize_i4(w, group)
    assert q.shape == (rows, (cols + 127) // 128 * 64) and scale.shape == (rows, (cols + group - 1) // group)
    want_q, want_scale = quantised(w, group)
    assert np.array_equal(unpack(q, cols), want_q)
    assert np.array_equal(scale.cpu().numpy(), want_scale)
    # nothing in the places past the rows' ends, no zero with a sign
    assert np.array_equal(q.cpu().numpy(), pack(want_q))


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_halves_go_to_the_even_number(slz, dtype):  # noqa: F811
    for top in (14.0, 3.5, 98.0, 14 * 2.0 ** -9):
        w = torch.zeros((1, 64), dtype=WIDE)
        w[0, :14] = (torch.arange(14, dtype=WIDE) - 6.5) * top / 7
        w[0, 20] = top
        w = w.to(dtype).cuda()
        q, _ = slz.quantize_i4(w, 64)
        assert unpack(q, 64)[0, :14].tolist() == [-6, -6, -4, -4, -2, -2, 0, 0, 2, 2, 4, 4, 6, 6]
    if dtype == torch.float32:                         # the neighbours of a half
        one = torch.full((1,), 7.0)
        for n in range(7):
            half = torch.full((1,), n + 0.5)
            w = torch.cat((one, half, torch.nextafter(half, one * 0), torch.nextafter(half, one * 2), -half)).reshape(1, 5).cuda()
            even = n + n % 2
            assert unpack(slz.quantize_i4(w, 32)[0], 5)[0].tolist() == [7, even, n, n + 1, -even]


def test_quantize_of_groups_without_a_scale(slz):  # noqa: F811
    for dtype in TYPES:
        w = randn((6, 200), 1, dtype)
        w[1] = 0
        w[2, 3] = float("inf")
        w[3, 199] = float("nan")
        w[4] = -0.0
        w[5, 64:] = float("-inf")
        q, scale = slz.quantize_i4(w, 64)
        want_q, want_scale = quantised(w, 64)
        assert np.array_equal(unpack(q, 200), want_q) and np.array_equal(scale.cpu().numpy(), want_scale, equal_nan=True)
        assert np.array_equal(q.cpu().numpy(), pack(want_q))
    for scale in (1e-38, 3e-45, 3e38):                 # 7 / top or 14 w is not a 32-bit number
        w = torch.tensor([[1.0, -0.5, 0.25, 0.08, 0.07, 0.0]], device="cuda", dtype=WIDE) * scale
        for dtype in (torch.float32, torch.bfloat16):
            q, s = slz.quantize_i4(w.to(dtype), 32)
            want_q, want_s = quantised(w.to(dtype), 32)
            assert np.array_equal(unpack(q, 6), want_q) and np.array_equal(s.cpu().numpy(), want_s)
    q, scale = slz.quantize_i4(torch.empty((3, 0), device="cuda"))
    assert q.shape == (3, 0) and scale.shape == (3, 0)
    q, scale = slz.quantize_i4(torch.empty((0, 200), device="cuda"))
    assert q.shape == (0, 128) and scale.shape == (0, 2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 33), (5, 128), (2, 1001), (200, 784)])
def test_values_are_scale_times_entry(slz, dtype, rows, cols):  # noqa: F811
    for group in GROUPS:
        q, packed, scale = weights(rows, cols, group, rows + cols)
        want = (torch.from_numpy(q).cuda().float() * scale.repeat_interleave(group, 1)[:, :cols]).to(dtype)
        assert torch.equal(slz.values_i4(packed, scale, cols, group, dtype), want)
    assert slz.values_i4(packed[:0], scale[:0], cols, group, dtype).shape == (0, cols)


# ---- product ------------------------------------------------------------------------------------------------------------------------
PRODUCTS = [(1, 1, 1), (1, 5, 16), (2, 3, 31), (1, 128, 784), (1, 1000, 1024), (3, 777, 130), (5, 64, 33), (7, 1001, 1555), (16, 256, 4096), (17, 100, 64), (32, 128, 784), (33, 65, 129),
            (48, 500, 640), (64, 1000, 4099), (65, 16, 500), (100, 3000, 300), (127, 129, 127), (128, 128, 128), (130, 257, 255), (257, 300, 1000), (500, 1100, 70), (1030, 520, 33), (5, 2, 20001)]


def bounds(x, w, want, dtype, count, rounded=True):
    """Of a product of x (rows) and w (rows), summed over `count`."""
    terms = x.abs() @ w.abs().t()
    operand = 2.0 ** -21 if dtype == torch.float32 else U[dtype] if rounded else 0.0
    return terms * ((count + 8) * 2.0 ** -24 + 1.01 * operand) + want.abs() * 1.01 * U[dtype] + LEAST[dtype]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_linear_is_the_formula(slz, dtype, m, n, k):  # noqa: F811
    for group in GROUPS:
        x = randn((m, k), m + n, dtype, slack=(m + n) % 3)
        q, packed, scale = weights(n, k, group, k)
        w = values(q, scale, group)
        y = slz.linear_i4(x, packed, scale, group)
        assert y.dtype == dtype
        want = x.to(WIDE) @ w.t()
        inside(y, want, bounds(x.to(WIDE), w, want, dtype, k), "y, group %d" % group)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [1, 3, 17, 70, 300])
def test_linear_with_weights_and_inputs_from_the_middle_of_others(slz, dtype, m):  # noqa: F811
    n, k, group = 150, 700, 64
    q, packed, scale = weights(n + 9, k + 256, group, 3)
    x = randn((m, k), 4, dtype, slack=1, skip=3)
    rows, cols = slice(5, 5 + n), slice(128, 128 + k)
    part = packed[rows, 64:64 + (k + 127) // 128 * 64]
    part_scale = scale[rows, 2:2 + (k + group - 1) // group]
    y = slz.linear_i4(x, part, part_scale, group)
    whole = torch.from_numpy(pack(q[rows, cols])).cuda()                           # zeros past the rows' ends, where part has other entries
    assert torch.equal(y, slz.linear_i4(x.contiguous(), whole, part_scale.contiguous(), group))
    dy = randn((m, n), 5, dtype)
    for p, t in zip(slz.linear_i4_grad(dy, x, part, part_scale, group), slz.linear_i4_grad(dy, x.contiguous(), whole, part_scale.contiguous(), group)):
        assert torch.equal(p, t)
    assert torch.equal(slz.values_i4(part, part_scale, k, group, dtype), slz.values_i4(whole, part_scale.contiguous(), k, group, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [1, 4, 20, 64, 130, 600])
def test_linear_keeps_infinities_and_nan_where_they_belong(slz, dtype, m):  # noqa: F811
    n, k, group = 70, 333, 32
    q, packed, scale = weights(n, k, group, 7, dead=False)
    # what lies past the ends of the rows, of the scales' rows and of x's rows has no influence
    wide = torch.cat((packed, torch.full((n, 64), 0xff, dtype=torch.uint8, device="cuda")), 1)
    last = pack(np.full((n, 384 - 333), 0))            # the codes past the last column, all set
    assert last.shape[1] == 64
    k_all = np.concatenate((q, np.full((n, 384 - k), -7)), 1)
    wide[:, :192] = torch.from_numpy(pack(k_all)).cuda()
    scales = torch.cat((scale, torch.full((n, 1), float("nan"), device="cuda")), 1)
    x = randn((m, k), 8, dtype, slack=3)
    x.as_strided((m, 3), (k + 3, 1), k).fill_(float("nan"))
    want = slz.linear_i4(x.contiguous(), packed, scale, group)
    got = slz.linear_i4(x, wide[:, :192], scales[:, :-1], group)
    assert torch.isfinite(want).all() and torch.equal(got, want)
    # a NaN scale is its column's, an infinity in x its row's
    scales[9, 2] = float("nan")
    got = slz.linear_i4(x, wide[:, :192], scales[:, :-1], group)
    rest = [i for i in range(n) if i != 9]
    assert torch.isnan(got[:, 9]).all() and torch.equal(got[:, rest], want[:, rest])
    x[m // 2, 40] = float("inf")
    got = slz.linear_i4(x, packed, scale, group)
    others = [i for i in range(m) if i != m // 2]
    assert not torch.isfinite(got[m // 2]).any() and torch.equal(got[others], want[others])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m, n, k", [(1, 70, 333), (7, 70, 333), (20, 70, 333), (90, 70, 1333), (2500, 90, 333)])
def test_linear_of_an_infinity_is_the_formulas(slz, dtype, m, n, k):  # noqa: F811
    # an infinity times an entry is that infinity, its negative, or NaN for an entry of zero; the other columns of its row and the other rows have no part in it
    q, packed, scale = weights(n, k, 64, 17, dead=False)
    x = randn((m, k), 18, dtype)
    x[m // 2, 40] = float("inf")
    x[m - 1, k - 1] = float("-inf")
    got = slz.linear_i4(x, packed, scale, 64).float().cpu().numpy()
    want = np.zeros((m, n))
    with np.errstate(invalid="ignore"):
        want[m // 2] += np.inf * q[:, 40]
        want[m - 1] += -np.inf * q[:, k - 1]
    lost = ~np.isfinite(want)
    np.testing.assert_array_equal(got[lost], want[lost])
    assert np.isfinite(got[~lost]).all()


def test_products_without_elements(slz):  # noqa: F811
    _, q, scale = weights(6, 100, 64, 1)
    for m in (1, 40, 300):
        x = randn((m, 100), 1)
        assert slz.linear_i4(x[:0], q, scale, 64).shape == (0, 6)
        assert slz.linear_i4(x, q[:0], scale[:0], 64).shape == (m, 0)
        y = slz.linear_i4(x[:, :0], q[:, :0], scale[:, :0], 64)
        assert y.shape == (m, 6) and (y == 0).all()
    x, dy = randn((5, 100), 2), randn((5, 6), 3)
    dx, dw = slz.linear_i4_grad(dy[:0], x[:0], q, scale, 64)
    assert dx.shape == (0, 100) and dw.shape == (6, 100) and (dw == 0).all()
    dx, dw = slz.linear_i4_grad(dy[:, :0], x, q[:0], scale[:0], 64)
    assert dw.shape == (0, 100) and dx.shape == (5, 100) and (dx == 0).all()
    dx, dw = slz.linear_i4_grad(dy, x[:, :0], q[:, :0], scale[:, :0], 64)
    assert dx.shape == (5, 0) and dw.shape == (6, 0)


def test_linear_past_four_gib(slz):  # noqa: F811
    n, k, group = (1 << 20) + 77, 8192, 128            # rows of 4 KiB: the last ones lie past 2^32 bytes
    gen = torch.Generator(device="cuda").manual_seed(1)
    packed = torch.randint(0, 256, (n, k // 2), dtype=torch.uint8, device="cuda", generator=gen)
    scale = torch.rand((n, k // group), device="cuda", generator=gen) * 0.01
    for m in (1, 20):
        x = randn((m, k), m, torch.bfloat16)
        y = slz.linear_i4(x, packed, scale, group)
        for rows in (slice(0, 64), slice(n - 100, n)):
            w = values(unpack(packed[rows], k), scale[rows], group)
            want = x.to(WIDE) @ w.t()
            inside(y[:, rows], want, bounds(x.to(WIDE), w, want, torch.bfloat16, k), "y")


# ---- gradient -----------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_linear_grad_is_the_formula(slz, dtype, m, n, k):  # noqa: F811
    group = GROUPS[(m + n + k) % 3]
    x, dy = randn((m, k), m + n, dtype, slack=(m + n) % 3), randn((m, n), k, dtype, slack=k % 2)
    q, packed, scale = weights(n, k, group, k)
    w = values(q, scale, group)
    dx, dw = slz.linear_i4_grad(dy, x, packed, scale, group)
    assert dx.dtype == dw.dtype == dtype
    d = dy.to(WIDE)
    want = d @ w
    inside(dx, want, bounds(d, w.t(), want, dtype, n), "dx")
    want = d.t() @ x.to(WIDE)
    inside(dw, want, bounds(d.t(), x.to(WIDE).t(), want, dtype, m, rounded=False), "dw")
    only_x, none = slz.linear_i4_grad(dy, x, packed, scale, group, need_w=False)
    assert none is None and torch.equal(only_x, dx)
    none, only_w = slz.linear_i4_grad(dy, x, packed, scale, group, need_x=False)
    assert none is None and torch.equal(only_w, dw)


def test_linear_grad_against_differences(slz):  # noqa: F811
    # the product is linear in x and in each value, so differences have no error but rounding
    m, n, k, group = 4, 6, 70, 32
    q, packed, scale = weights(n, k, group, 3, dead=False)
    x, dy = randn((m, k), 1), randn((m, n), 2)
    dx, dw = slz.linear_i4_grad(dy, x, packed, scale, group)

    def loss(a, p):
        return (slz.linear_i4(a, p, scale, group).to(WIDE) * dy.to(WIDE)).sum()

    w = values(q, scale, group)
    # each sum of n k products in 32 bits, twice
    noise = 2 * (k + n + 8) * 2.0 ** -23 * ((x.to(WIDE).abs() @ w.abs().t()) * dy.to(WIDE).abs()).sum().item()
    for i, j in ((0, 0), (2, 33), (3, 69)):
        up, down = x.clone(), x.clone()
        up[i, j] += 0.5
        down[i, j] -= 0.5
        step = (up[i, j] - down[i, j]).to(WIDE).item()
        assert abs((loss(up, packed) - loss(down, packed)).item() / step - dx[i, j].item()) <= 2 * noise / step
    for i, j in ((0, 0), (4, 40), (5, 69)):
        up, down = q.copy(), q.copy()
        up[i, j], down[i, j] = 7, -7
        step = 14 * scale[i, j // group].to(WIDE).item()
        diff = (loss(x, torch.from_numpy(pack(up)).cuda()) - loss(x, torch.from_numpy(pack(down)).cuda())).item()
        assert abs(diff - step * dw[i, j].item()) <= 4 * noise


@pytest.mark.parametrize("dtype", TYPES)
def test_values_of_any_scale(slz, dtype):  # noqa: F811
    # one term a sum, so that each value shows by itself; scales from 1 down to 2^-24, and all of them far from 1
    n, k = 72, 96
    rng = np.random.default_rng(5)
    q = rng.integers(-7, 8, (n, k))
    packed = torch.from_numpy(pack(q)).cuda()
    for far in (1.0, 2.0 ** -60, 2.0 ** 40):
        s = (far * 1.37 * 2.0 ** (-torch.arange(n, device="cuda", dtype=WIDE) / 3)).float()[:, None].expand(n, 3).contiguous()
        w = values(q, s, 32)
        x = torch.zeros((n, n), device="cuda", dtype=dtype)
        x.fill_diagonal_(200.0)
        want = 200 * w
        value = U[dtype] if dtype != torch.float32 else 2.0 ** -21
        top = torch.finfo(dtype).max
        bound = want.abs() * 1.01 * (value + U[dtype] + 8 * 2.0 ** -24) + LEAST[dtype]
        dx = slz.linear_i4_grad(x, torch.zeros((n, k), device="cuda", dtype=dtype), packed, s, 32, need_w=False)[0]
        fits = want.abs() < 0.99 * top
        inside(torch.where(fits, dx, 0), torch.where(fits, want, 0), bound, "dx")
        for m in (1, 20, 200):                         # the product: rows of x with a single entry
            x = torch.zeros((m, k), device="cuda", dtype=dtype)
            at = torch.arange(m, device="cuda") * 5 % k
            x[torch.arange(m, device="cuda"), at] = 200.0
            want_y = 200 * w.t()[at]
            fits = want_y.abs() < 0.99 * top
            y = slz.linear_i4(x, packed, s, 32)
            bound = want_y.abs() * 1.01 * (value + U[dtype] + 8 * 2.0 ** -24) + LEAST[dtype]
            inside(torch.where(fits, y, 0), torch.where(fits, want_y, 0), bound, "y of %d" % m)


@pytest.mark.parametrize("dtype", TYPES)
def test_small_inputs_are_not_lost(slz, dtype):  # noqa: F811
    # inputs below the type's smallest ordinary number, times scales that bring the results back
    n, k, group = 40, 256, 64
    q, packed, _ = weights(n, k, group, 3)
    scale = torch.full((n, k // group), 2.0 ** 13 if dtype == torch.float16 else 2.0 ** 120, device="cuda")
    w = values(q, scale, group)
    step = 2.0 ** -24 if dtype == torch.float16 else 2.0 ** -133
    for m in (1, 5, 40, 200):
        x = (torch.randint(-60, 61, (m, k), device="cuda", generator=torch.Generator(device="cuda").manual_seed(m)).to(WIDE) * step).to(dtype)
        assert (x != 0).any() and x.abs().max() < torch.finfo(dtype).tiny
        want = x.to(WIDE) @ w.t()
        inside(slz.linear_i4(x, packed, scale, group), want, bounds(x.to(WIDE), w, want, dtype, k), "y")


def test_the_c_entries_write_between_other_data(slz):  # noqa: F811
    # rows of everything further apart than they are long, and results at addresses that are no multiples of 16 bytes; what lies between stays
    import ctypes
    from paper_2504_17785_amd.clear import SlzI4Shape, _TYPES
    L = slz.lib()
    stream = torch.cuda.current_stream().cuda_stream
    for dtype in TYPES:
        for m, n, k, group in ((1, 50, 333, 32), (40, 70, 260, 64), (300, 90, 129, 128), (3000, 3200, 72, 64)):
            e = torch.finfo(dtype).bits // 8
            w = randn((n, k), 1, dtype, slack=3)
            blocks, groups = (k + 127) // 128, (k + group - 1) // group
            q = torch.full((n, blocks * 64 + 48), 0xaa, dtype=torch.uint8, device="cuda")
            scale = torch.full((n, groups + 2), -5.0, device="cuda")
            assert L.slz_quantize_i4(w.data_ptr(), _TYPES[dtype], n, k, k + 3, group, q.data_ptr(), q.shape[1], scale.data_ptr(), groups + 2, stream) == 0
            want_q, want_scale = slz.quantize_i4(w, group)
            assert torch.equal(q[:, :blocks * 64], want_q) and (q[:, blocks * 64:] == 0xaa).all()
            assert torch.equal(scale[:, :groups], want_scale) and (scale[:, groups:] == -5).all()

            def room(rows, cols):
                t = torch.full((rows * (cols + 5) + 1,), 7.0, dtype=dtype, device="cuda")
                return t, t[1:].view(rows, cols + 5)[:, :cols], t.data_ptr() + e

            whole, values, at = room(n, k)
            assert L.slz_values_i4(q.data_ptr(), q.shape[1], scale.data_ptr(), groups + 2, group, n, k, at, _TYPES[dtype], k + 5, stream) == 0
            assert torch.equal(values, slz.values_i4(want_q, want_scale, k, group, dtype))
            values.fill_(7.0)
            assert (whole == 7).all()
            x, dy = randn((m, k), 2, dtype, slack=1), randn((m, n), 3, dtype, slack=2)
            sh = SlzI4Shape(m, n, k, _TYPES[dtype], group, k + 1, q.shape[1], groups + 2, n + 5)
            need = ctypes.c_size_t(0)
            assert L.slz_linear_i4_workspace(ctypes.byref(sh), x.data_ptr(), ctypes.byref(need)) == 0
            ws = torch.empty(need.value + 256, dtype=torch.uint8, device="cuda")
            whole, y, at = room(m, n)
            assert L.slz_linear_i4(ctypes.byref(sh), x.data_ptr(), q.data_ptr(), scale.data_ptr(), at, ws.data_ptr(), need.value, stream) == 0
            assert torch.equal(y, slz.linear_i4(x, want_q, want_scale, group))
            y.fill_(7.0)
            assert (whole == 7).all()
            sh.ld_y = n + 2
            assert L.slz_linear_i4_grad_workspace(ctypes.byref(sh), dy.data_ptr(), x.data_ptr(), ctypes.byref(need)) == 0
            ws = torch.empty(need.value + 256, dtype=torch.uint8, device="cuda")
            (whole_x, dx, at_x), (whole_w, dw, at_w) = room(m, k), room(n, k)
            assert L.slz_linear_i4_grad(ctypes.byref(sh), dy.data_ptr(), x.data_ptr(), q.data_ptr(), scale.data_ptr(), at_x, k + 5, at_w, k + 5, ws.data_ptr(), need.value, stream) == 0
            want_x, want_w = slz.linear_i4_grad(dy, x, want_q, want_scale, group)
            assert torch.equal(dx, want_x) and torch.equal(dw, want_w)
            dx.fill_(7.0)
            dw.fill_(7.0)
            assert (whole_x == 7).all() and (whole_w == 7).all()


def test_more_rows_than_a_launch_of_small_tiles_takes(slz):  # noqa: F811
    m, n, k, group = (1 << 27) + 5, 4, 8, 32
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((m, k), device="cuda", generator=gen, dtype=torch.bfloat16)
    q, packed, scale = weights(n, k, group, 2)
    w = values(q, scale, group)
    y = slz.linear_i4(x, packed, scale, group)
    for rows in (slice(0, 1000), slice(m // 2, m // 2 + 1000), slice(m - 1000, m)):
        want = x[rows].to(WIDE) @ w.t()
        inside(y[rows], want, bounds(x[rows].to(WIDE), w, want, torch.bfloat16, k), "y")


# ---- all ----------------------------------------------------------------------------------------------------------------------------
def calls(slz):  # noqa: F811
    out = []
    for dtype, m in ((torch.bfloat16, 1), (torch.float16, 9), (torch.float32, 40), (torch.bfloat16, 200), (torch.float16, 700)):
        _, q, scale = weights(300, 500, 64, m)
        x, dy = randn((m, 500), m, dtype, slack=m % 2), randn((m, 300), m + 1, dtype)
        out += [lambda x=x, q=q, scale=scale: slz.linear_i4(x, q, scale, 64), lambda dy=dy, x=x, q=q, scale=scale: slz.linear_i4_grad(dy, x, q, scale, 64),
                lambda x=x: slz.quantize_i4(x, 64), lambda q=q, scale=scale, dtype=dtype: slz.values_i4(q, scale, 500, 64, dtype)]
    return out


def test_the_same_inputs_give_the_same_bits_on_any_stream(slz):  # noqa: F811
    for call in calls(slz):
        first = [t.clone() for t in leaves(call())]
        torch.cuda.synchronize()
        s, r = torch.cuda.Stream(), torch.cuda.Stream()
        again = []
        for _ in range(3):                             # two streams at once
            for stream in (s, r):
                with torch.cuda.stream(stream):
                    again.append(leaves(call()))
        torch.cuda.synchronize()
        for got in again:
            for p, q in zip(first, got):
                assert torch.equal(p, q)


def test_calls_can_be_captured_and_replayed(slz):  # noqa: F811
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


def test_the_binding_refuses(slz):  # noqa: F811
    x, dy = randn((8, 200), 1), randn((8, 10), 2)
    _, q, scale = weights(10, 200, 64, 3)
    with pytest.raises(TypeError):
        slz.linear_i4(x.double(), q, scale, 64)
    with pytest.raises(TypeError):
        slz.linear_i4(x, q.to(torch.int8), scale, 64)
    with pytest.raises(TypeError):
        slz.linear_i4(x, q, scale.half(), 64)
    with pytest.raises(TypeError):
        slz.values_i4(q, scale, 200, 64, torch.int8)
    with pytest.raises(TypeError):
        slz.linear_i4_grad(dy.half(), x, q, scale, 64)
    for group in (0, 16, 96, 256):
        with pytest.raises(ValueError):
            slz.linear_i4(x, q, scale, group)
        with pytest.raises(ValueError):
            slz.quantize_i4(x, group)
    with pytest.raises(ValueError):
        slz.linear_i4(x, q, scale, 32)                 # scales of other groups
    with pytest.raises(ValueError):
        slz.linear_i4(x[:, :100], q, scale, 64)
    with pytest.raises(ValueError):
        slz.linear_i4(x, q, scale[:9], 64)
    with pytest.raises(ValueError):
        slz.linear_i4(x.t(), q, scale, 64)
    with pytest.raises(ValueError):
        slz.linear_i4(x, q.t(), scale, 64)
    with pytest.raises(ValueError):
        slz.linear_i4_grad(dy[:, :9], x, q, scale, 64)
    with pytest.raises(ValueError):
        slz.linear_i4_grad(dy[:7], x, q, scale, 64)
    with pytest.raises(ValueError):
        slz.values_i4(q, scale, -1, 64)
    with pytest.raises(slz.SlzError):                  # rows that do not lie on 16 bytes
        slz.linear_i4(x[:, :128], torch.zeros((10, 72), dtype=torch.uint8, device="cuda")[:, 4:68], scale[:, :2], 64)
    with pytest.raises(slz.SlzError):
        slz.linear_i4(x[:, :128], torch.zeros((10, 72), dtype=torch.uint8, device="cuda")[:, :64], scale[:, :2], 64)


def test_a_backward_pass_does_not_skip_what_autograd_cannot_do(slz):  # noqa: F811
    x = randn((4, 128), 1).requires_grad_()
    _, q, scale = weights(6, 128, 128, 2)
    with pytest.raises(RuntimeError, match="linear_i4"):
        slz.linear_i4(x, q, scale).sum().backward()
    with pytest.raises(RuntimeError, match="quantize_i4"):
        slz.quantize_i4(x)[1].sum().backward()
