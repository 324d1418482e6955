"""A training step with 4-bit layers (examples/clear_step.py) taken apart: each product, the loss and each gradient against its formula in 64 bits on the very inputs that the step gave it, so that
a bound is one operation's and small against the result; and the head's gradient against differences along itself."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_clear import TYPES, WIDE, check_ce, inside, slz  # noqa: E402,F401
from tests.test_gpu_clear_i4 import bounds, unpack, values  # noqa: E402
from tests.test_gpu_clear_i4_step import network  # noqa: E402


def told_apart(want, bound):
    """Zeros, a part left out or another sign would not be inside."""
    assert bound.norm() < 0.1 * want.norm(), (bound.norm() / want.norm()).item()


@pytest.mark.parametrize("dtype", TYPES)
def test_each_operation_of_a_step(slz, dtype):  # noqa: F811
    example, net, x, labels = network(dtype=dtype)
    seen = []

    class Recorder(example.Mlp):
        def layer_grad(self, dy, kept, need_x):
            out = super().layer_grad(dy, kept, need_x)
            seen.append((dy, out))
            return out

    net.__class__ = Recorder
    loss, count, grads, kept = net.gradients(x, labels)
    seen.reverse()                                     # in the order of the layers
    assert len(seen) == len(kept) == 2 and count == (labels != -100).sum()

    h = x.to(dtype)
    for i, ((h_kept, q, scale), y) in enumerate(kept):
        assert torch.equal(h_kept, h)
        want_q, want_scale = slz.quantize_i4(net.weights[i], net.GROUP)
        assert torch.equal(q, want_q) and torch.equal(scale, want_scale)
        w = values(unpack(q, h.shape[1]), scale, net.GROUP)
        want = h.to(WIDE) @ w.t()
        bound = bounds(h.to(WIDE), w, want, dtype, h.shape[1], rounded=False)
        told_apart(want, bound)
        inside(y, want, bound, "y of layer %d" % i)
        h = y.relu()

    # the head: its own check against the formula, and the same bits here
    counts = (labels != -100).float()
    head_loss, _, dh, dw = check_ce(slz, h, net.weights[-1].to(dtype), labels, counts / counts.sum())
    assert torch.equal(loss, head_loss.sum()) and torch.equal(grads[-1], dw)

    for i in reversed(range(2)):
        (h_kept, q, scale), y = kept[i]
        dy, (dx, dw) = seen[i]
        assert torch.equal(dy, dh * (y > 0))
        d, a = dy.to(WIDE), h_kept.to(WIDE)
        want = d.t() @ a
        bound = bounds(d.t(), a.t(), want, dtype, d.shape[0], rounded=False)
        told_apart(want, bound)
        inside(dw, want, bound, "dw of layer %d" % i)
        assert torch.equal(grads[i], dw)
        if i == 0:
            assert dx is None
            break
        w = values(unpack(q, a.shape[1]), scale, net.GROUP)
        want = d @ w
        bound = bounds(d, w.t(), want, dtype, d.shape[1])
        told_apart(want, bound)
        inside(dx, want, bound, "dx of layer %d" % i)
        dh = dx


def test_the_heads_gradient_against_differences_along_itself(slz):  # noqa: F811
    # the head's weights are not quantised; along the gradient, as long as that the logits move by 1 at most
    _, net, x, labels = network()
    _, _, grads, kept = net.gradients(x, labels)
    g, at = grads[-1].to(WIDE), net.weights[-1].clone()
    h = kept[-1][1].relu().to(WIDE)
    reach = (h @ g.t()).abs().amax()
    step, both, ways = 2.0 ** -4, [], []
    for sign in (1, -1):
        net.weights[-1] = (at.to(WIDE) + sign * step / reach * g).float()
        ways.append(net.weights[-1].to(WIDE))
        loss, count, _, _ = net.gradients(x, labels)
        both.append((loss / count).item())
    d = ways[0] - ways[1]
    slope = (g * d).sum().item()
    # A logit is off by its terms' magnitudes times what 72 products in 32 bits and their missing pieces make, a loss by two logits and the roundings of its logarithm, 32 bits of each
    terms = h.abs() @ torch.maximum(ways[0].abs(), ways[1].abs()).t()
    off = terms.amax(1) * (80 * 2.0 ** -24 + 2.0 ** -21)
    loss_off = (2 * off + 8 * 2.0 ** -24 * (terms.amax(1) + math.log(10))).mean().item() + 64 * 2.0 ** -24 * max(both)
    # the gradient by the same and its sums
    p = torch.softmax(h @ at.to(WIDE).t(), 1)
    hot = torch.nn.functional.one_hot(labels.clamp(min=0), 10).to(WIDE)
    counts = (labels != -100).to(WIDE)[:, None]
    slope_off = ((((p * (2 * off[:, None] + 2.0 ** -18) + (p + hot) * 2.0 ** -19) * counts / counts.sum()).t() @ h.abs()) * d.abs()).sum().item()
    # the third derivative of a log-sum whose terms move by -1 to 1 is a third central moment over a range of 2: at most 2^3 / (6 sqrt 3); the difference takes step^3 / 3 of it
    bend = 8 / (6 * math.sqrt(3)) * step ** 3 / 3
    allowed = 2 * loss_off + slope_off + bend
    assert allowed < 0.02 * slope, (allowed, slope)
    assert abs(both[0] - both[1] - slope) <= allowed, (both[0] - both[1], slope, allowed)
