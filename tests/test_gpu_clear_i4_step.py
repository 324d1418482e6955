"""4-bit layers, the loss, clipped gradients and answers as a program uses them together (examples/clear_step.py): the gradients against the same network in 64 bits, with the values that its
layers stand for and the rectifiers that were on, and against differences."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_clear import U, WIDE, slz  # noqa: E402,F401
from tests.test_gpu_clear_i4 import unpack, values  # noqa: E402


def network(bits=4, dtype=torch.float32, **kw):
    import examples.clear_step as example
    net = example.Mlp(widths=(200, 96, 72, 10), dtype=dtype, bits=bits, **kw)
    x, labels = example.synthetic(64, inner=200, seed=11)
    labels[5] = -100
    return example, net, x, labels


def reference(net, x, labels, kept):
    """Gradients in 64 bits, and for each the same formula of magnitudes: what roundings are relative to."""
    ws = [values(unpack(q, w.shape[1]), scale, net.GROUP) for ((_, q, scale), _), w in zip(kept, net.weights)] + [net.weights[-1].to(net.dtype).to(WIDE)]
    hs, mags = [x.to(net.dtype).to(WIDE)], [x.to(net.dtype).to(WIDE).abs()]
    for w, (_, y) in zip(ws, kept):
        on = (y > 0).to(WIDE)
        hs.append((hs[-1] @ w.t()) * on)
        mags.append((mags[-1] @ w.abs().t()) * on)
    p = torch.softmax(hs[-1] @ ws[-1].t(), 1)
    counts = labels != -100
    hot = torch.zeros_like(p)
    hot[counts, labels[counts]] = 1
    g = (p - hot) * counts[:, None] / counts.sum()
    # z is off by its terms' magnitudes times the unit below, and p by p times that
    off = (mags[-1] @ ws[-1].abs().t()).amax(1, keepdim=True)
    m = (p + hot) * counts[:, None] / counts.sum() * (1 + 2 * off)
    grads, bounds = [], []
    for i in reversed(range(len(ws))):
        grads.insert(0, g.t() @ hs[i])
        bounds.insert(0, m.t() @ mags[i])
        if i:
            on = (kept[i - 1][1] > 0).to(WIDE)
            g, m = (g @ ws[i]) * on, (m @ ws[i].abs()) * on
    return grads, bounds


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_of_a_4_bit_network(slz, dtype):  # noqa: F811
    _, net, x, labels = network(dtype=dtype)
    _, _, grads, kept = net.gradients(x, labels)
    want, bounds = reference(net, x, labels, kept)
    # along a gradient's way lie three products forward and up to three back: each sums up to 200 terms in 32 bits (f32: operands to 2^-21 of their magnitudes) and rounds operands and results to the type
    unit = 6 * (202 * 2.0 ** -24 + 2.0 ** -21) if dtype == torch.float32 else 6 * (202 * 2.0 ** -24 + 3 * U[dtype])
    for got, t, b in zip(grads, want, bounds):
        assert got.shape == t.shape and got.dtype == dtype
        assert ((got.to(WIDE) - t).abs() <= unit * b + 1e-30).all(), ((got.to(WIDE) - t).abs() / b).max()


def test_gradients_against_differences(slz):  # noqa: F811
    # the head's weights are not quantised: the mean loss along a direction of them
    example, net, x, labels = network()
    loss, count, grads, _ = net.gradients(x, labels)
    d = torch.randn(net.weights[-1].shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    step, at = 2.0 ** -6, net.weights[-1].clone()
    both = []
    for sign in (1, -1):
        net.weights[-1] = at + sign * step * d
        loss, count, _, _ = net.gradients(x, labels)
        both.append((loss / count).item())
    slope = (grads[-1].to(WIDE) * d.to(WIDE)).sum().item()
    # the third derivative of the log-sum along d is at most (2 |z'|)^3, z' = h d; the losses of up to some tens have 24 bits, summed over 64 tokens
    _, _, _, kept = net.gradients(x, labels)
    reach = (kept[-1][1].relu().to(WIDE) @ d.to(WIDE).t()).abs().amax().item()
    assert abs((both[0] - both[1]) / (2 * step) - slope) <= (2 * reach) ** 3 * step ** 2 / 6 + 64 * max(both) * 2.0 ** -23 / step


def test_a_step_clips_its_gradients_before_it_uses_them(slz):  # noqa: F811
    _, net, x, labels = network()
    _, again, _, _ = network(clip=0.01)
    _, _, grads, _ = net.gradients(x, labels)
    norm = math.sqrt(sum((g.to(WIDE) ** 2).sum().item() for g in grads))
    assert norm > 0.01
    again.step(x, labels)
    f = 0.01 / (norm + 1e-6)
    for m, g in zip(again.momentum, grads):            # momentum begins at zero
        assert ((m - f * g).abs() <= f * g.abs() * 4 * 2.0 ** -24 + 1e-30).all()


@pytest.mark.parametrize("bits", [4, 8])
def test_the_example_runs_and_answers(slz, bits):  # noqa: F811
    example, _, _, _ = network()
    losses, right, one, among = example.train(steps=3, bits=bits, clip=1.0)
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses) and 0 <= right <= 1
    # an input alone and among others: two layers' sums in another order, rounded to bf16 in between and at the end
    assert ((one - among).abs() <= 8 * U[torch.bfloat16] * (among.abs().amax() + 1)).all()
