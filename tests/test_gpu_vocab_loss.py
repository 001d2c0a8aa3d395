"""Softmax cross entropy over a vocabulary and its gradients against the formulas in 64 bits and against differences."""
import math

import pytest

import paper_2501_09849_b200 as cdl

pytestmark = pytest.mark.gpu

TYPES = {"bf16": (cdl.CDL_BF16, "bfloat16", 2.0 ** -8), "f16": (cdl.CDL_F16, "float16", 2.0 ** -11)}


def up(n, m=8):
    return -(-n // m) * m


def problem(torch, T, V, D, kind, seed, ignore=0.2, pad=0, size=1.0):
    g = torch.Generator().manual_seed(seed)
    dt = getattr(torch, TYPES[kind][1])
    h = torch.full((T, up(D) + pad), float("nan"), dtype=dt)           # what lies between the rows is not read
    w = torch.full((V, up(D) + pad), float("nan"), dtype=dt)
    h[:, :D] = (torch.randn(T, D, generator=g) * size).to(dt)
    w[:, :D] = (torch.randn(V, D, generator=g) * (1.5 / math.sqrt(D))).to(dt)
    y = torch.randint(0, V, (T,), generator=g)
    drop = torch.rand(T, generator=g) < ignore
    y = torch.where(drop, torch.tensor([-100, -1, V, 2 ** 40])[torch.randint(0, 4, (T,), generator=g)], y)
    gl = torch.randn(T, generator=g) / max(T, 1)
    gl = torch.where(drop, torch.full_like(gl, float("nan")), gl)      # not read where there is no label
    return h.cuda(), w.cuda(), y.cuda(), gl.cuda()


def run(torch, h, w, y, gl, T, V, D, kind, need=("dh", "dw"), stream=None):
    code, dtype, _ = TYPES[kind]
    dt = getattr(torch, dtype)
    nb = cdl.cdl_vocab_loss_workspace_bytes(T, V, D, 1)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    loss, lse = torch.full((T,), -7.0, device="cuda"), torch.full((T,), -7.0, device="cuda")
    cdl.cdl_vocab_loss_fwd(h, h.stride(0), w, w.stride(0), code, y, T, V, D, loss, lse, ws, nb, stream=stream)
    dh = torch.full((T, up(D) + 8), 9.0, dtype=dt, device="cuda") if "dh" in need else None
    dw = torch.full((V, up(D) + 8), 9.0, dtype=dt, device="cuda") if "dw" in need else None
    cdl.cdl_vocab_loss_bwd(h, h.stride(0), w, w.stride(0), code, y, lse, gl, T, V, D, dh, up(D) + 8, dw, up(D) + 8, ws, nb, stream=stream)
    cdl.cdl_workspace_status(ws)
    for d in (dh, dw):
        assert d is None or bool((d[:, D:] == 9.0).all())
    return loss, lse, None if dh is None else dh[:, :D], None if dw is None else dw[:, :D]


def reference(torch, h, w, y, gl, T, V, D):
    H, W = h[:, :D].double(), w[:, :D].double()
    logits = H @ W.t()
    lse = torch.logsumexp(logits, 1)
    counts = (y >= 0) & (y < V)
    at = torch.where(counts, y, torch.zeros_like(y))
    loss = torch.where(counts, lse - logits.gather(1, at[:, None])[:, 0], torch.zeros_like(lse))
    p = torch.exp(logits - lse[:, None])
    g = torch.where(counts, gl.double(), torch.zeros_like(lse))
    hot = torch.zeros_like(p)
    hot.scatter_(1, at[:, None], 1.0)
    dl = g[:, None] * (p - hot)
    return H, W, logits, lse, counts, loss, p, g, dl


def check(torch, got, h, w, y, gl, T, V, D, kind):
    loss, lse, dh, dw = got
    H, W, logits, lse_r, counts, loss_r, p, g, dl = reference(torch, h, w, y, gl, T, V, D)
    u = TYPES[kind][2]
    # a logit: D / 16 tensor-core sums, each good to 2^-23 of the terms' magnitudes
    mag = H.abs() @ W.abs().t()
    e_logit = (mag.max(1).values + 1e-30) * (D / 16 + 1) * 2.0 ** -23
    # the exponent's argument is rounded at the logit's and the maximum's size, the exponential is good to 2^-21, sums are binary32
    size = logits.abs().max(1).values + lse_r.abs()
    e_lse = e_logit + size * 2.0 ** -22 + 2.0 ** -20
    assert bool(((lse.double() - lse_r).abs() <= e_lse + lse_r.abs() * 2.0 ** -23).all())
    assert bool(((loss.double() - loss_r).abs() <= e_lse + e_logit + size * 2.0 ** -22).all())
    assert bool((loss[~counts] == 0).all())
    rel = (e_logit + e_lse + size * 2.0 ** -22 + 2.0 ** -20)[:, None]         # of a probability
    # dl is rounded to 16 bits; in binary16 its smallest step is 2^-24 of a scale that puts the largest |dloss| above 2^14
    e_dl = dl.abs() * u + g.abs()[:, None] * p * rel * (1 + u) + (float(g.abs().max()) * 2.0 ** -38 if kind == "f16" else 1e-40)
    for out, ref, err, terms in ((dh, dl @ W, e_dl @ W.abs(), dl.abs() @ W.abs()), (dw, dl.t() @ H, e_dl.t() @ H.abs(), dl.abs().t() @ H.abs())):
        if out is None:
            continue
        n = V if out.shape[0] == T and out is dh else T
        tol = err + terms * (n / 16 + 8) * 2.0 ** -23 + ref.abs() * u + (2.0 ** -24 if kind == "f16" else 0.0)
        bad = (out.double() - ref).abs() - tol
        assert bool((bad <= 0).all()), float(((out.double() - ref).abs() / tol).max())


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("T,V,D,pad", [(1, 1, 1, 0), (1, 1000, 64, 0), (2, 129, 8, 8), (5, 257, 65, 0), (64, 3000, 200, 0), (127, 511, 136, 16), (128, 256, 64, 0),
                                       (129, 255, 72, 0), (256, 640, 512, 0), (300, 5000, 333, 0), (777, 2049, 100, 0), (1000, 9001, 264, 0)])
def test_loss_and_gradients(kind, T, V, D, pad):
    import torch
    h, w, y, gl = problem(torch, T, V, D, kind, T + V + D, pad=pad)
    check(torch, run(torch, h, w, y, gl, T, V, D, kind), h, w, y, gl, T, V, D, kind)


@pytest.mark.parametrize("kind", list(TYPES))
def test_several_pieces_of_the_vocabulary(kind):
    import torch
    T, V, D = 5000, 20011, 72                    # dl of a piece is bounded: the vocabulary is taken in several pieces
    h, w, y, gl = problem(torch, T, V, D, kind, 3)
    check(torch, run(torch, h, w, y, gl, T, V, D, kind), h, w, y, gl, T, V, D, kind)


def test_many_pieces_and_a_short_last_one():
    import torch
    T, V, D = 16500, 4200, 64                    # pieces of 2048 words: the last has 104
    h, w, y, gl = problem(torch, T, V, D, "bf16", 4)
    check(torch, run(torch, h, w, y, gl, T, V, D, "bf16"), h, w, y, gl, T, V, D, "bf16")


def test_one_gradient_alone_is_the_same():
    import torch
    T, V, D = 200, 1500, 96
    h, w, y, gl = problem(torch, T, V, D, "bf16", 5)
    both = run(torch, h, w, y, gl, T, V, D, "bf16")
    assert torch.equal(both[2], run(torch, h, w, y, gl, T, V, D, "bf16", need=("dh",))[2])
    assert torch.equal(both[3], run(torch, h, w, y, gl, T, V, D, "bf16", need=("dw",))[3])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = run(torch, h, w, y, gl, T, V, D, "bf16")
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(both, again))


@pytest.mark.parametrize("kind", list(TYPES))
def test_every_position_ignored(kind):
    import torch
    T, V, D = 140, 700, 64
    h, w, y, gl = problem(torch, T, V, D, kind, 7, ignore=2.0)
    loss, lse, dh, dw = run(torch, h, w, y, gl, T, V, D, kind)
    assert bool((loss == 0).all()) and bool((dh == 0).all()) and bool((dw == 0).all()) and bool(torch.isfinite(lse).all())


@pytest.mark.parametrize("kind", list(TYPES))
def test_large_logits_and_tiny_gradients(kind):
    import torch
    T, V, D = 150, 900, 128
    h, w, y, gl = problem(torch, T, V, D, kind, 8, ignore=0.0, size=40.0)      # logits in the hundreds: one word takes all
    gl = gl * 1e-6                                                               # a mean over a very large batch
    check(torch, run(torch, h, w, y, gl, T, V, D, kind), h, w, y, gl, T, V, D, kind)


@pytest.mark.parametrize("T", [1, 2, 7, 150])
def test_rows_that_outgrow_their_first_columns(T):
    """Logits that rise by hundreds along the vocabulary, fall, or begin at -infinity: the base of a row's sums has to follow."""
    import torch
    V, D = 1200, 64
    h, w, y, gl = problem(torch, T, V, D, "bf16", 12, ignore=0.0)
    h[:, :D] = 0
    w[:, :D] = 0
    h[:, 0] = 1.0
    h[:, 1] = torch.where(torch.arange(T, device="cuda") % 2 == 0, 1.0, -1.0).to(h.dtype)
    w[:, 1] = torch.linspace(-300, 300, V, device="cuda").to(w.dtype)
    w[:, 0] = torch.randn(V, generator=torch.Generator().manual_seed(2)).to(w.dtype).cuda()
    w[700:, 1] = 0.0
    check(torch, run(torch, h, w, y, gl, T, V, D, "bf16"), h, w, y, gl, T, V, D, "bf16")
    w[:500, 1] = float("-inf")                            # even rows: the first words cannot be; odd rows: +infinity
    y = torch.full_like(y, 900)
    loss, lse, _, _ = run(torch, h, w, y, gl, T, V, D, "bf16", need=("dh",))
    logits = h[::2, :D].double() @ w[:, :D].double().nan_to_num(neginf=-1e300).t()
    ref = torch.logsumexp(logits, 1)
    assert bool(((lse[::2].double() - ref).abs() <= 2.0 ** -18 * ref.abs()).all())
    assert bool((torch.isnan(lse[1::2]) | torch.isinf(lse[1::2])).all())


def test_non_finite_rows_stay_in_their_rows():
    import torch
    T, V, D = 130, 400, 64
    h, w, y, gl = problem(torch, T, V, D, "bf16", 9, ignore=0.0)
    clean = run(torch, h, w, y, gl, T, V, D, "bf16")
    h2 = h.clone()
    h2[3, 5] = float("nan")
    bad = run(torch, h2, w, y, gl, T, V, D, "bf16")
    keep = torch.arange(T, device="cuda") != 3
    assert torch.equal(bad[0][keep], clean[0][keep]) and torch.equal(bad[2][keep], clean[2][keep])
    assert bool(torch.isnan(bad[0][3])) and bool(torch.isnan(bad[1][3]))


def test_gradient_against_differences():
    import torch
    T, V, D = 90, 600, 80
    h, w, y, gl = problem(torch, T, V, D, "bf16", 10)
    _, _, dh, dw = run(torch, h, w, y, gl, T, V, D, "bf16")
    H, W = h[:, :D].double(), w[:, :D].double()
    counts = (y >= 0) & (y < V)
    g = torch.where(counts, gl.double(), torch.zeros(T, device="cuda", dtype=torch.float64))
    at = torch.where(counts, y, torch.zeros_like(y))

    def total(H, W):
        l = H @ W.t()
        return (g * (torch.logsumexp(l, 1) - l.gather(1, at[:, None])[:, 0])).sum()

    gen = torch.Generator().manual_seed(1)
    for which, grad in ((0, dh), (1, dw)):
        d = torch.randn(grad.shape, generator=gen, dtype=torch.float64).cuda()
        e = 1e-4
        ends = [total(H + s * e * d, W) if which == 0 else total(H, W + s * e * d) for s in (1, -1)]
        diff = float(ends[0] - ends[1]) / (2 * e)
        got = float((grad.double() * d).sum())
        # two roundings to 16 bits (dl and the result), independent between entries: far below their worst case of 2 * 2^-8
        assert abs(diff - got) <= 2 * 2.0 ** -8 * float((grad.double().abs() * d.abs()).sum())


def test_no_positions():
    import torch
    V, D = 300, 72
    w = torch.randn(V, D, device="cuda").to(torch.bfloat16)
    dw = torch.full((V, 80), 3.0, dtype=torch.bfloat16, device="cuda")
    assert cdl.cdl_vocab_loss_fwd(None, 0, w, D, cdl.CDL_BF16, None, 0, V, D, None, None) == 0
    assert cdl.cdl_vocab_loss_bwd(None, 0, w, D, cdl.CDL_BF16, None, None, None, 0, V, D, None, 0, dw, 80) == 0
    assert bool((dw[:, :D] == 0).all()) and bool((dw[:, D:] == 3.0).all())
