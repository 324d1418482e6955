"""Clipping of matrices that lie between each other's rows: apart, they are clipped; where they meet, refused."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_clear import randn, slz  # noqa: E402,F401
from tests.test_gpu_clear_clip import factor, near, wide_norm  # noqa: E402


def test_rows_at_different_distances_that_do_not_meet(slz):  # noqa: F811
    g = randn((40, 64), 1)
    kept = g.clone()
    parts = [g[:, :10], g[::2, 20:30], g[1::2, 20:30], g[::3, 30:41], g[1::3, 30:41], g[2::3, 30:41], g[:20, 50:], g[20::4, 50:]]
    mine = [p.clone() for p in parts]
    norm = slz.clip_by_norm(parts, 0.5)
    near(norm, wide_norm(mine))
    f = factor(norm.item(), 0.5)
    for p, k in zip(parts, mine):
        assert torch.equal(p, k * f)
    # what is in none of them stays
    assert torch.equal(g[:, 10:20], kept[:, 10:20]) and torch.equal(g[:, 41:50], kept[:, 41:50])
    for first in (21, 22, 23):
        assert torch.equal(g[first::4, 50:], kept[first::4, 50:])


def test_rows_at_different_distances_that_meet_are_refused(slz):  # noqa: F811
    g, h = randn((40, 64), 2), randn((19, 64), 3)
    kept = g.clone()
    for grads, out in (([g[:, :21], g[::2, 20:30]], None), ([g[::2, 20:30], g[::3, 29:41]], None), ([g[1::2, :10], g[39:, :5]], None), ([g[:19], h], [g[1:20], h]),
                       ([g[:19]], [g.as_strided((19, 64), (64, 1), 1)])):
        with pytest.raises(slz.SlzError):
            slz.clip_by_norm(grads, 1e-3, out=out)
    assert torch.equal(g, kept)
