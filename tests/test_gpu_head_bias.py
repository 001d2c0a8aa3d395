"""The head's bias is trained: its gradient is the column sums of dY, eagerly and in a recorded step."""
import pytest

from paper_2501_09849_b200.head import HeadStep

pytestmark = pytest.mark.gpu


def step(torch, T=200, D=136, V=900, bias=True):
    g = torch.Generator().manual_seed(2)
    s = HeadStep(torch, T, D, V, p=0.1, seed=3, bias=bias)
    s.x.copy_(torch.randn(T, D, generator=g))
    s.labels.copy_(torch.randint(0, 20, (T,), generator=g))
    s.w1.copy_(torch.randn(D, D, generator=g) / D ** 0.5)
    s.w2.copy_(torch.randn(V, D, generator=g) / D ** 0.5)
    return s


@pytest.mark.parametrize("recorded", [False, True])
def test_gradient_of_the_bias(recorded):
    import torch
    s = step(torch)
    if recorded:
        graph = s.capture()
        s.db1.fill_(float("nan"))
        graph.replay()
    else:
        s.run()
    ref = s.dy.double().sum(0)
    # binary32 sums of 200 numbers
    assert bool(((s.db1.double() - ref).abs() <= s.dy.double().abs().sum(0) * 200 * 2.0 ** -24).all())
    assert bool((ref != 0).any())


def test_descent_along_the_bias_alone():
    import torch
    s = step(torch)
    s.run()
    first, small = float(s.loss.mean()), float((s.db1 ** 2).sum())
    rate = 0.05 / small
    s.b1.sub_(rate * s.db1)
    s.run()
    # the loss falls by rate |db1|^2 = 0.05 to first order; 8-bit products and the second order leave half of it
    assert float(s.loss.mean()) < first - 0.025


def test_no_bias_no_gradient():
    import torch
    s = step(torch, bias=False)
    s.run()
    assert s.b1 is None and s.db1 is None
