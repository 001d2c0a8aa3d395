"""The vocabulary loss' gradient at positions that the model predicts with near certainty: the label's entry of dl is the distance of a
probability from 1, which must keep its relative accuracy although log-sum-exp is a binary32 number of the logits' size.

Every confident row has dimensions of its own, so that the gradient of the weights holds that row's dl alone, one product per entry."""
import math

import pytest

import paper_2501_09849_b200 as cdl

pytestmark = pytest.mark.gpu

TYPES = {"bf16": (cdl.CDL_BF16, "bfloat16", 2.0 ** -9), "f16": (cdl.CDL_F16, "float16", 2.0 ** -11)}      # half a step, relative
ROWS = 24


def problem(torch, T, V, kind, size, seed):
    """ROWS positions of losses from 5e-6 to 0.3 among logits of `size`, the others without a label."""
    g = torch.Generator().manual_seed(seed)
    dt = getattr(torch, TYPES[kind][1])
    D = 8 * ROWS
    h, w = torch.randn(T, D, generator=g).to(dt), torch.zeros(V, D, dtype=dt)
    h[:ROWS] = 0
    rows = torch.randperm(T, generator=g)[:ROWS] if T > ROWS else torch.arange(ROWS)
    h[rows] = 0
    y = torch.full((T,), -100)
    words = torch.randint(0, V, (ROWS,), generator=g)
    words[0], words[1] = 0, V - 1
    y[rows] = words
    for t in range(ROWS):
        loss = 5e-6 * (0.3 / 5e-6) ** (t / (ROWS - 1))
        h[rows[t], 8 * t], h[rows[t], 8 * t + 1] = 16.0, 1.0
        w[:, 8 * t] = size / 16.0
        w[:, 8 * t + 1] = -(math.log((V - 1) / loss) + 0.5 * torch.randn(V, generator=g)).to(dt)
        w[words[t], 8 * t + 1] = 0
        w[:, 8 * t + 2] = torch.randn(V, generator=g).to(dt)           # not part of the logits: shows dl in dH
    return h.cuda(), w.cuda(), y.cuda(), rows.cuda(), words.cuda(), D


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("size", [12.0, 25.0, 300.0])
@pytest.mark.parametrize("T,V", [(24, 1000), (100, 2500), (300, 3001), (2100, 17000), (2101, 33333)])
def test_label_entries_keep_their_relative_accuracy(kind, size, T, V):
    import torch
    h, w, y, rows, words, D = problem(torch, T, V, kind, size, T + V)
    code, _, u = TYPES[kind]
    gl = torch.full((T,), 512.0, device="cuda")
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    nb = cdl.cdl_vocab_loss_workspace_bytes(T, V, D, 1)
    ws = torch.full((nb,), 255, dtype=torch.uint8, device="cuda")          # (as floats: NaN)
    cdl.cdl_vocab_loss_fwd(h, D, w, D, code, y, T, V, D, loss, lse, ws, nb)
    ws.fill_(255)
    cdl.cdl_vocab_loss_bwd(h, D, w, D, code, y, lse, gl, T, V, D, dh, D, dw, D, ws, nb)
    cdl.cdl_workspace_status(ws)
    W = w.double()
    logits = h[rows].double() @ W.t()
    other = logits.clone()
    other[torch.arange(ROWS), words] = -math.inf
    ref_lse = torch.logsumexp(logits, 1)
    entry = -torch.exp(torch.logsumexp(other, 1) - ref_lse)
    p = torch.exp(other - ref_lse[:, None])
    # logits and lse to 2^-23 and 2^-24 of their terms' size, the exponent's argument rounded once at theirs, the exponential 2^-21; with
    # several pieces of the vocabulary an entry that is not small may be 2^-10 off
    rel = (h[rows].double().abs() @ W.abs().t()).max(1).values * 4 * 2.0 ** -23 + 2.0 ** -20
    loose = 2.0 ** -10 if T > 2000 else 0.0
    own = 8 * torch.arange(ROWS, device="cuda")
    got = dw[words, own + 1].double() / 512.0                              # dl and the result rounded to 16 bits
    off = (got / entry - 1).abs()
    assert bool((off <= 2 * u * (1 + u) + rel + loose).all()), off.tolist()
    got = dh[rows, own + 2].double()
    ref = 512.0 * ((p * W[:, own + 2].t()).sum(1) + entry * W[words, own + 2])
    size_dl = 512.0 * ((p * W[:, own + 2].t().abs()).sum(1) + entry.abs() * W[words, own + 2].abs())
    floor = V * 512.0 * 2.0 ** -38 * 4 if kind == "f16" else 0.0           # binary16's smallest step of dl, weights below 4
    assert bool(((got - ref).abs() <= size_dl * (2 * u + rel + loose) + floor).all())
    assert bool((dh[y == -100] == 0).all())


def test_many_confident_rows_are_reproducible():
    """Rows are put together in any order, their results must not depend on it."""
    import torch
    T, V, D = 3000, 12000, 64
    g = torch.Generator().manual_seed(5)
    w = (torch.randn(V, D, generator=g) * 0.64).to(torch.bfloat16).cuda()
    y = torch.randint(0, V, (T,), generator=g).cuda()
    h = (w[y].double() * (0.3 + 1.2 * torch.rand(T, 1, generator=g).cuda().double())).to(torch.bfloat16)        # from certain to open
    gl = torch.full((T,), 1.0 / T, device="cuda")
    outs = []
    for _ in range(4):
        loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        dh, dw = torch.empty_like(h), torch.empty_like(w)
        nb = cdl.cdl_vocab_loss_workspace_bytes(T, V, D, 1)
        ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
        cdl.cdl_vocab_loss_fwd(h, D, w, D, cdl.CDL_BF16, y, T, V, D, loss, lse, ws, nb)
        cdl.cdl_vocab_loss_bwd(h, D, w, D, cdl.CDL_BF16, y, lse, gl, T, V, D, dh, D, dw, D, ws, nb)
        cdl.cdl_workspace_status(ws)
        outs.append((loss, lse, dh, dw))
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))
    lse64 = torch.logsumexp(h.double() @ w.double().t(), 1)
    p = torch.exp(h.double() @ w.double().t() - lse64[:, None])
    small = 1 - p[torch.arange(T), y]
    assert int((small < 1e-3).sum()) > 300 and int((small > 0.1).sum()) > 300
    p[torch.arange(T), y] = 0
    p[torch.arange(T), y] = -p.sum(1)
    ref = p @ w.double() / T
    # two independent roundings to 16 bits, row by row
    assert bool(((outs[0][2].double() - ref).norm(dim=1) <= 2 * 2.0 ** -8 * ref.norm(dim=1)).all())


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("T,V,D,seed", [(1, 4644, 1184, 1), (1, 700, 2000, 2), (2, 3000, 1504, 3), (3, 3000, 1504, 4), (200, 2000, 1600, 5)])
def test_label_entries_of_improbable_words_are_minus_one(kind, T, V, D, seed):
    """Logits in the hundreds, labels of next to no probability: the entry does not take part in the errors of the other probabilities."""
    import torch
    code, dtype, u = TYPES[kind]
    dt = getattr(torch, dtype)
    g = torch.Generator().manual_seed(seed)
    h = (40 * torch.randn(T, D, generator=g)).to(dt)
    w = (torch.randn(V, D, generator=g) * (1.5 / math.sqrt(D))).to(dt)
    logits = h.double() @ w.double().t()
    p = torch.softmax(logits, 1)
    y = torch.empty(T, dtype=torch.int64)
    taken = set()
    for t in range(T):                       # an improbable word of its own, which no other row gives any probability
        for v in torch.randperm(V, generator=g).tolist():
            if float(p[:, v].max()) < 1e-12 and v not in taken:
                y[t] = v
                taken.add(v)
                break
    assert len(taken) == T
    h, w, y = h.cuda(), w.cuda(), y.cuda()
    gl = torch.full((T,), 1.0, device="cuda")
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    nb = cdl.cdl_vocab_loss_workspace_bytes(T, V, D, 1)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    cdl.cdl_vocab_loss_fwd(h, D, w, D, code, y, T, V, D, loss, lse, ws, nb)
    cdl.cdl_vocab_loss_bwd(h, D, w, D, code, y, lse, gl, T, V, D, dh, D, dw, D, ws, nb)
    cdl.cdl_workspace_status(ws)
    # dl is -1, which has no rounding; the weights' gradient at the label is -h but for the other rows' 1e-12
    assert bool(((dw[y].double() + h.double()).abs() <= h.double().abs() * u + 1e-9 * T).all())
