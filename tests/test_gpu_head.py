"""The language-model operators together, as a training step of an output head uses them: each stage of the step against the
64-bit value of its own inputs, and a descent."""
import pytest

import paper_2501_09849_b200 as cdl
from paper_2501_09849_b200.head import HeadStep

pytestmark = pytest.mark.gpu


def filled(torch, T, D, V, p, bias=False, seed=3):
    g = torch.Generator().manual_seed(seed)
    s = HeadStep(torch, T, D, V, p=p, seed=11, bias=bias)
    s.x.copy_(torch.randn(T, D, generator=g))
    s.labels.copy_(torch.randint(0, V, (T,), generator=g))
    s.labels[1] = -100
    s.w1.copy_(torch.randn(D, D, generator=g) / D ** 0.5)
    s.w2.copy_(torch.randn(V, D, generator=g) / D ** 0.5)
    if bias:
        s.b1.copy_(torch.randn(D, generator=g))
    return s


def values(codes, scales, rows, cols, mode):
    s = scales.double()
    s = s if mode == "rows" else s.repeat_interleave(128, 1)[:, :rows]
    return codes[:, :cols].double() * s.t().repeat_interleave(128, 1)[:, :cols]


@pytest.mark.parametrize("T,D,V,bias", [(2, 8, 30, False), (130, 264, 1001, True), (515, 384, 3000, False)])
def test_every_stage(T, D, V, bias):
    import torch
    s = filled(torch, T, D, V, 0.25, bias)
    s.run(first_index=40)
    cdl.cdl_workspace_status(s.ws)
    half = 2.0 ** -8
    x, w = values(s.xc, s.xs, T, D, "rows"), values(s.w1c, s.w1s, D, D, "blocks")
    y = x @ w.t() + (s.b1.double() if bias else 0.0)
    size = x.abs() @ w.abs().t() + (s.b1.double().abs() if bias else 0.0)
    # products of 8-bit codes: bounds of the product's own test (four sums of 2^-22 per block of 128, binary32 between blocks)
    slack = 4 * 2.0 ** -22 + (-(-max(T, D) // 128) + 12) * 2.0 ** -24
    assert bool(((s.y.double() - y).abs() <= size * slack + y.abs() * half).all())
    kept = (s.h.double() - s.x.double()).abs() > 1e-9
    h = s.y.double() / 0.75 + s.x.double()
    assert bool(((s.h.double() - torch.where(kept, h, s.x.double())).abs() <= h.abs() * half + 2.0 ** -20 * (h.abs() + s.x.double().abs())).all())
    # the loss of these hidden states, and its gradients
    logits = s.h.double() @ s.w2.double().t()
    counts = s.labels >= 0
    at = s.labels.clamp(min=0)[:, None]
    lse = torch.logsumexp(logits, 1)
    loss = torch.where(counts, lse - logits.gather(1, at)[:, 0], torch.zeros_like(lse))
    assert float((s.loss.double() - loss).abs().max()) <= 1e-4
    d = torch.exp(logits - lse[:, None]).scatter_add(1, at, -torch.ones_like(at, dtype=torch.float64)) * (counts.double() / T)[:, None]
    for got, ref in ((s.dh, d @ s.w2.double()), (s.dw2, d.t() @ s.h.double())):
        # two independent roundings to 16 bits (dl and the result)
        assert float((got.double() - ref).norm()) <= 2 * half * float(ref.norm())
    # dropout again, on the gradient: nothing passes where the forward pass dropped
    again = torch.empty_like(s.h)
    ones = torch.ones_like(s.h)
    cdl.cdl_dropout(ones, D, None, 0, again, D, cdl.CDL_BF16, T, D, 0.25, 11, 40)
    mask = again != 0
    assert bool((s.dy[~mask] == 0).all())
    assert bool(((s.dy.double() - s.dh.double() / 0.75).abs()[mask] <= (s.dh.double().abs() / 0.75 * (half + 2.0 ** -20))[mask]).all())
    g, gt = values(s.gc, s.gs, T, D, "rows"), values(s.gct, s.gst, D, T, "rows")
    wt, xt = values(s.w1ct, s.w1st, D, D, "blocks"), values(s.xct, s.xst, D, T, "rows")
    assert torch.equal(wt, w.t())
    dx = g @ wt.t()
    tol = g.abs() @ wt.abs().t() * slack + dx.abs() * half + (dx + s.dh.double()).abs() * half + 2.0 ** -20 * s.dh.double().abs()
    assert bool(((s.dx.double() - dx - s.dh.double()).abs() <= tol).all())
    assert bool(((s.dw1.double() - gt @ xt.t()).abs() <= gt.abs() @ xt.abs().t() * slack).all())


def test_recorded_step_equals_the_issued_one():
    import torch
    s = filled(torch, 200, 136, 700, 0.1)
    s.run()
    names = ("loss", "lse", "dh", "dw2", "dx", "dw1")
    issued = [getattr(s, n).clone() for n in names]
    for n in names:
        getattr(s, n).zero_()
    s.capture().replay()
    for n, ref in zip(names, issued):
        assert torch.equal(getattr(s, n), ref), n


def test_descent():
    import torch
    T, D, V = 256, 128, 500
    s = filled(torch, T, D, V, 0.1)
    s.labels.clamp_(min=0)
    w2 = s.w2.float()
    first = None
    for k in range(25):
        s.w2.copy_(w2)
        s.run(first_index=k * T * D)
        first = float(s.loss.mean()) if first is None else first
        s.w1.sub_(0.5 * s.dw1)
        w2.sub_(0.5 * T * s.dw2.float())
    assert float(s.loss.mean()) < 0.5 * first
