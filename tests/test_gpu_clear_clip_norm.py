"""Clipping by a given norm that autograd follows: its outputs depend on the norm, and autograd would not know."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_clear import slz  # noqa: E402,F401


def test_a_norm_with_a_gradient_is_refused_while_autograd_records(slz):  # noqa: F811
    p = torch.ones((8,), device="cuda", requires_grad=True)
    norm = (p * p).sum().sqrt()
    g = torch.ones((8,), device="cuda")
    with pytest.raises(RuntimeError, match="clip_by_norm"):
        slz.clip_by_norm([g], 1.0, norm=norm)
    assert (g == 1).all()
    with torch.no_grad():
        slz.clip_by_norm([g], 1.0, norm=norm)
    assert (g < 1).all()
    slz.clip_by_norm([g], 1.0, norm=norm.detach())
