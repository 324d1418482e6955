"""Gradients clipped by their norm (include/silenzio_clear.h) against the formula: squares and their sum have 64 bits, so the norm is the one in 64 bits
rounded once, and given the norm every element is the formula's bit for bit."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_clear import TYPES, WIDE, randn, slz  # noqa: E402,F401

EPS = 1e-6


def wide_norm(grads):
    return math.sqrt(math.fsum((g.to(WIDE) ** 2).sum().item() for g in grads))


def factor(norm, max_norm, eps=EPS):
    limit = np.float64(np.float32(norm)) + np.float64(np.float32(eps))
    top = np.float64(np.float32(max_norm))
    return float(np.float32(top / limit)) if limit > top else 1.0 if limit <= top else float("nan")


def near(norm, want):
    # some thousand additions in 64 bits on either side, and one rounding to 32
    assert abs(norm.item() - want) <= want * (1.01 * 2.0 ** -24 + 2.0 ** -40) + 2.0 ** -149, (norm.item(), want)


def mixed(shapes, seed, std=1.0):
    return [randn(s, seed + i, TYPES[i % 3], std=std) if len(s) else randn((1,), seed + i, TYPES[i % 3], std=std).reshape(()) for i, s in enumerate(shapes)]


def check(slz, grads, max_norm, eps=EPS, in_place=False):  # noqa: F811
    kept = [g.clone() for g in grads]
    out = [torch.empty_like(g) for g in grads]
    norm = slz.clip_by_norm(grads, max_norm, eps, out=None if in_place else out)
    got = grads if in_place else out
    near(norm, wide_norm(kept))
    assert torch.equal(norm, slz.grad_norm(kept))
    f = factor(norm.item(), max_norm, eps)
    for g, k, o in zip(grads, kept, got):
        assert torch.equal(o, (k.float() * f).to(k.dtype))
        assert in_place or torch.equal(g, k)
    return f


SHAPES = [
    [(1,)],
    [()],
    [(7,), (3, 5), (0,), (2, 0, 4), (1, 1, 1)],
    [(128, 784), (128,), (64, 128), (64,), (10, 64), (10,)],
    [(2047,), (2048,), (2049,), (4097, 3)],
    [(i % 37 + 1, i % 11) for i in range(63)],
    [(i % 37 + 1, 5) for i in range(64)],
    [(i % 37 + 1, 3) for i in range(65)],
    [(i % 5 + 1, i % 3) for i in range(240)],
    [(i * 97 % 4000 + 1,) for i in range(161)],
    [(i % 5 + 1,) for i in range(4097)],
    [(3000, 1001), (5,), (4096, 4096), (1,)],
]


@pytest.mark.parametrize("shapes", SHAPES, ids=range(len(SHAPES)))
@pytest.mark.parametrize("in_place", [False, True])
def test_clip_is_the_formula(slz, shapes, in_place):  # noqa: F811
    for std, clips in ((1.0, True), (1e-4, False)):
        grads = mixed(shapes, 3, std)
        # beyond one where the standard deviation is, unless there are few elements
        f = check(slz, grads, 0.01 if clips else 1e4, in_place=in_place)
        assert (f < 1) == clips


@pytest.mark.parametrize("dtype", TYPES)
def test_clip_of_any_address_and_distance(slz, dtype):  # noqa: F811
    base = randn((40, 301), 1, dtype)
    flat = randn((5000,), 2, dtype)
    grads = [base[:, :7], base[:, 7:100], base[3:9, 100:301], flat[1:2500], flat[2501:2502], randn((33, 64), 3, dtype, slack=3, skip=1), base[20:21, 100:130]]
    kept_base, kept_flat = base.clone(), flat.clone()
    kept = [g.clone() for g in grads]
    norm = slz.clip_by_norm(grads, 0.5)
    near(norm, wide_norm(kept))
    f = factor(norm.item(), 0.5)
    for g, k in zip(grads, kept):
        assert torch.equal(g, (k.float() * f).to(dtype))
    # what lies between them stays
    assert torch.equal(base[9:20, 100:], kept_base[9:20, 100:]) and torch.equal(base[:3, 100:], kept_base[:3, 100:])
    assert flat[0] == kept_flat[0] and flat[2500] == kept_flat[2500] and torch.equal(flat[2502:], kept_flat[2502:])
    # more of them than a launch takes in its arguments, rows further apart among them
    many = [randn((7, 5 + i % 3), 10 + i, dtype, slack=i % 4, skip=i % 2) for i in range(150)]
    kept = [g.clone() for g in many]
    norm = slz.clip_by_norm(many, 0.5)
    near(norm, wide_norm(kept))
    assert all(torch.equal(g, (k.float() * factor(norm.item(), 0.5)).to(dtype)) for g, k in zip(many, kept))
    # from rows further apart into one run, and the other way round
    g = randn((33, 64), 4, dtype, slack=2)
    run, rows = torch.zeros((33, 64), dtype=dtype, device="cuda"), torch.zeros((33, 70), dtype=dtype, device="cuda")
    norm = slz.clip_by_norm([g], 0.5, out=[run])
    slz.clip_by_norm([g.contiguous()], 0.5, out=[rows[:, 3:67]])
    want = (g.float() * factor(norm.item(), 0.5)).to(dtype)
    assert torch.equal(run, want) and torch.equal(rows[:, 3:67], want) and (rows[:, :3] == 0).all() and (rows[:, 67:] == 0).all()


def test_clip_of_special_values(slz):  # noqa: F811
    for scale in (1e-30, 1e30):                        # squares leave 32 bits
        check(slz, [randn((500, 30), 1) * scale, randn((77,), 2) * scale], scale, 0.0)
    g = randn((100,), 3) * 3e37                        # the norm does not
    assert check(slz, [g], 1.0) < 1
    big = [torch.full((1000,), 3e38, device="cuda")]   # it does: f is 0
    norm = slz.clip_by_norm(big, 1.0)
    assert norm.item() == float("inf") and (big[0] == 0).all()
    for bad in (float("nan"), float("inf")):
        grads = [randn((100,), 4), randn((5, 6), 5, torch.bfloat16)]
        kept = [t.clone() for t in grads]
        grads[0][7] = bad
        norm = slz.clip_by_norm(grads, 1.0)
        assert math.isnan(norm.item()) if math.isnan(bad) else norm.item() == bad
        if math.isnan(bad):
            assert all(torch.isnan(t).all() for t in grads)
        else:                                          # f = 0, and 0 times the infinity
            assert torch.isnan(grads[0][7]) and (grads[1] == 0).all() and torch.isnan(grads[0]).sum() == 1
        again = [t.clone() for t in kept]
        slz.clip_by_norm(again, 1.0, norm=torch.tensor(bad, device="cuda"))
        assert torch.isnan(again[0]).all() if math.isnan(bad) else (again[0] == 0).all()
    zero = [torch.zeros((50,), device="cuda"), torch.full((3,), -0.0, device="cuda")]
    assert slz.clip_by_norm(zero, 0.0, 0.0).item() == 0
    assert (zero[0] == 0).all() and torch.signbit(zero[1]).all()
    # at the limit nothing changes, a little above it something does
    g = torch.ones((4,), device="cuda")
    slz.clip_by_norm([g], 2.0, 0.0)
    assert (g == 1).all()
    slz.clip_by_norm([g], 2.0, 1e-3)
    assert (g < 1).all()
    slz.clip_by_norm([g], float("inf"))
    check(slz, [randn((100,), 6)], 0.0)


def test_a_given_norm_is_taken(slz):  # noqa: F811
    grads = mixed([(300, 20), (77,), (5, 5, 5)], 8)
    for given in (0.25, 4.0, 1e9):
        norm = torch.tensor([given], device="cuda")
        out = [torch.empty_like(g) for g in grads]
        assert slz.clip_by_norm(grads, 1.0, norm=norm, out=out) is norm and norm.item() == np.float32(given)
        for g, o in zip(grads, out):
            assert torch.equal(o, (g.float() * factor(given, 1.0)).to(g.dtype))


def test_nothing_to_clip(slz):  # noqa: F811
    assert slz.grad_norm([]).item() == 0 and slz.clip_by_norm([], 1.0).item() == 0
    none = [torch.empty((0, 5), device="cuda"), torch.empty((0,), dtype=torch.float16, device="cuda")]
    assert slz.grad_norm(none).item() == 0 and slz.clip_by_norm(none, 1.0).item() == 0


def test_clip_of_more_elements_than_32_bits_count(slz):  # noqa: F811
    g = torch.full((65537, 32768), 0.5, dtype=torch.bfloat16, device="cuda")       # 2^31 + 2^15
    g[-1, -1] = 2.0 ** 14
    norm = slz.clip_by_norm([g], 1024.0, 0.0)
    near(norm, math.sqrt((g.numel() - 1) * 0.25 + 2.0 ** 28))
    f = factor(norm.item(), 1024.0, 0.0)
    want = (torch.tensor([0.5, 2.0 ** 14]) * f).bfloat16()
    assert g[-1, -1].item() == want[1] and g[0, 0].item() == want[0] and (g[65000:, :32767] == want[0].item()).all() and (g[32767] == want[0].item()).all()


def test_outputs_that_overlap_are_refused(slz):  # noqa: F811
    g, h = randn((20, 64), 1), randn((20, 64), 2)
    kept = g.clone()
    for grads, out in (([g, g], None), ([g, g[3:4]], None), ([g[:11], g[10:]], None), ([g, h], [h, g]), ([g], [g.view(-1)[1:].as_strided((19, 64), (64, 1))[:19]]),
                       ([g[:, :33], g[:, 32:]], None), ([g[:, :32], h], [g[:, 16:48], h]), ([g[:19], h], [g[1:], h]), ([h[:10], g], [g[5:15], g])):
        if out is not None and any(o.shape != x.shape for o, x in zip(out, grads)):
            continue
        with pytest.raises(slz.SlzError):
            slz.clip_by_norm(grads, 1e-3, out=out)
    assert torch.equal(g, kept)
    # the same gradient may be read twice, and columns of one matrix are apart
    near(slz.grad_norm([g, g]), math.sqrt(2) * wide_norm([g]))
    out = [torch.empty_like(g), torch.empty_like(g)]
    norm = slz.clip_by_norm([g, g], 1.0, out=out)
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], g * factor(norm.item(), 1.0))
    slz.clip_by_norm([g[:, :16], g[:, 16:40], g[:5, 40:], g[5, 40:], g[6:, 40:]], 1.0)
    # g counted once, all of it multiplied
    assert torch.equal(g, kept * factor(slz.grad_norm([kept]).item(), 1.0))


def test_the_same_bits_on_any_stream_and_replayed(slz):  # noqa: F811
    for shapes in (SHAPES[3], SHAPES[7]):
        grads = mixed(shapes, 5)
        out = [torch.empty_like(g) for g in grads]
        first_norm = slz.clip_by_norm(grads, 0.1, out=out).clone()
        first = [o.clone() for o in out]
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            again = [torch.empty_like(g) for g in grads]
            norm = slz.clip_by_norm(grads, 0.1, out=again)
        s.synchronize()
        assert torch.equal(norm, first_norm) and all(torch.equal(p, q) for p, q in zip(first, again))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            norm = slz.clip_by_norm(grads, 0.1, out=out)
        for i in range(4):
            for o in out:
                o.zero_()
            for g in grads:
                g.mul_(2)                              # other gradients: the norm and the factor follow
            want = [torch.empty_like(g) for g in grads]
            graph.replay()
            torch.cuda.synchronize()
            want_norm = slz.clip_by_norm(grads, 0.1, out=want)
            assert torch.equal(norm, want_norm) and all(torch.equal(p, q) for p, q in zip(want, out))


def test_the_binding_refuses(slz):  # noqa: F811
    g = randn((8, 32), 1)
    with pytest.raises(TypeError):
        slz.grad_norm([g.double()])
    with pytest.raises(TypeError):
        slz.grad_norm([g.cpu()])
    with pytest.raises(ValueError):
        slz.grad_norm([randn((4, 4, 8), 2)[:, :, ::2]])
    with pytest.raises(ValueError):
        slz.grad_norm([g.t()])
    with pytest.raises(ValueError):
        slz.grad_norm([g[:1].expand(4, 32)])
    with pytest.raises(ValueError):
        slz.clip_by_norm([g], 1.0, out=[])
    with pytest.raises(ValueError):
        slz.clip_by_norm([g], 1.0, out=[g.half()])
    with pytest.raises(ValueError):
        slz.clip_by_norm([g], 1.0, out=[torch.empty((32, 8), device="cuda")])
    with pytest.raises(TypeError):
        slz.clip_by_norm([g], 1.0, norm=torch.ones((2,), device="cuda"))
    with pytest.raises(TypeError):
        slz.clip_by_norm([g], 1.0, norm=torch.ones(()))
    for max_norm, eps in ((-1.0, EPS), (float("nan"), EPS), (1.0, -1e-3), (1.0, float("nan"))):
        with pytest.raises(slz.SlzError):
            slz.clip_by_norm([g], max_norm, eps)


def test_autograd_notices(slz):  # noqa: F811
    g = randn((8,), 1).requires_grad_()
    with pytest.raises(RuntimeError):
        slz.clip_by_norm([g], 1.0)
    with pytest.raises(RuntimeError, match="grad_norm"):
        slz.grad_norm([g]).backward()
    with torch.no_grad():
        slz.clip_by_norm([g], 1.0)
    # a tensor that a backward pass needs and that was clipped in between
    p, w = randn((8,), 2), randn((8,), 3).requires_grad_()
    y = (p * w).sum()
    slz.clip_by_norm([p], 1e-3)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
