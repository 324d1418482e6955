"""The shapes of tests/clear_i4_laid_out.py take the product of values that are laid out."""
from tests.clear_i4_laid_out import SHAPES
from tests.test_clear_cpu_i4_routes import route  # noqa: F401


def test_shapes_are_laid_out(route):  # noqa: F811
    for m, n, k in SHAPES:
        for group in (32, 64, 128):
            for wide in (False, True):
                assert route(m, n, k, group, wide)[0] == ("tiles", 0), (m, n, k, group, wide)
