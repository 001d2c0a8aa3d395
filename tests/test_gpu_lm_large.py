"""The language-model operators on tensors whose offsets pass 32 bits: sampled entries at the far end against 64-bit values."""
import pytest

import paper_2501_09849_b200 as cdl

pytestmark = pytest.mark.gpu


def test_quantizer_and_product_past_four_gigabytes():
    import torch
    N, K = 140000, 32768                       # 4.6e9 codes
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(N, K, dtype=torch.bfloat16, device="cuda")
    for r in range(0, N, 20000):
        x[r:r + 20000] = torch.randn(min(20000, N - r), K, generator=g, device="cuda", dtype=torch.bfloat16)
    codes = torch.empty(N, K, dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.empty(K // 128, N, device="cuda")
    ct = torch.empty(K, N, dtype=torch.float8_e4m3fn, device="cuda")
    st = torch.empty(-(-N // 128), K, device="cuda")
    cdl.cdl_fp8_quantize(x, K, cdl.CDL_BF16, N, K, cdl.CDL_FP8_ROWS, codes, K, scales, ct, N, st)
    for r in (0, 70001, N - 1):
        v = codes[r].double().view(-1, 128) * scales[:, r].double()[:, None]
        xr = x[r].double().view(-1, 128)
        # half a step of a code: 2^-4 of the value, or 2^-10 scales
        assert bool(((v - xr).abs() <= torch.maximum(xr.abs() * 2.0 ** -4, scales[:, r].double()[:, None] * 2.0 ** -10) * (1 + 2.0 ** -18)).all())
    for c in (0, 16383, K - 1):
        s = st[:, c].double().repeat_interleave(128)[:N]
        xc = x[:, c].double()
        assert bool(((ct[c].double() * s - xc).abs() <= torch.maximum(xc.abs() * 2.0 ** -4, s * 2.0 ** -10) * (1 + 2.0 ** -18)).all())
    del x, ct, st
    for M in (1, 3, 300):                      # every form of the product
        a = (torch.randn(M, K, generator=g, device="cuda") * 100).clamp_(-448, 448).to(torch.float8_e4m3fn)
        sa = torch.rand(K // 128, M, generator=g, device="cuda") + 0.5
        out = torch.empty(M, N, device="cuda")
        nb = cdl.cdl_fp8_matmul_workspace_bytes(M, N, K)
        ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
        cdl.cdl_fp8_matmul(a, K, sa, codes, K, scales, cdl.CDL_FP8_ROWS, M, N, K, out, N, cdl.CDL_F32, ws=ws, ws_bytes=nb)
        cdl.cdl_workspace_status(ws)
        at = torch.tensor([0, 1, 65535, 65536, 131072, N - 2, N - 1], device="cuda")
        A = a.double() * sa.t().double().repeat_interleave(128, 1)
        B = codes[at].double() * scales[:, at].t().double().repeat_interleave(128, 1)
        ref, size = A @ B.t(), A.abs() @ B.abs().t()
        # four sums of 2^-22 per block of 128 and binary32 between the 256 blocks
        assert bool(((out[:, at].double() - ref).abs() <= size * (4 * 2.0 ** -22 + (K // 128 + 12) * 2.0 ** -24)).all())


def test_vocabulary_past_four_gigabytes():
    import torch
    V, D = 1100000, 2048                       # 2.25e9 weights
    g = torch.Generator(device="cuda").manual_seed(2)
    w = torch.empty(V, D, dtype=torch.bfloat16, device="cuda")
    for r in range(0, V, 100000):
        w[r:r + 100000] = torch.randn(min(100000, V - r), D, generator=g, device="cuda", dtype=torch.bfloat16) * (1.5 / D ** 0.5)
    dw = torch.empty_like(w)
    for T in (1, 140):
        h = torch.randn(T, D, generator=g, device="cuda").to(torch.bfloat16)
        y = torch.randint(0, V, (T,), generator=g, device="cuda")
        y[0] = V - 1
        loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        gl = torch.full((T,), 1.0 / T, device="cuda")
        dh = torch.empty_like(h)
        nb = cdl.cdl_vocab_loss_workspace_bytes(T, V, D, True)
        ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
        cdl.cdl_vocab_loss_fwd(h, D, w, D, cdl.CDL_BF16, y, T, V, D, loss, lse, ws, nb)
        cdl.cdl_vocab_loss_bwd(h, D, w, D, cdl.CDL_BF16, y, lse, gl, T, V, D, dh, D, dw, D, ws, nb)
        cdl.cdl_workspace_status(ws)
        H = h.double()
        top, total, ref_dh = None, torch.zeros(T, dtype=torch.float64, device="cuda"), torch.zeros(T, D, dtype=torch.float64, device="cuda")
        for r in range(0, V, 100000):          # (logits of these weights are below 20: no maximum needed in 64 bits)
            W = w[r:r + 100000].double()
            e = torch.exp(H @ W.t())
            total += e.sum(1)
            ref_dh += e @ W
        ref_lse = torch.log(total)
        target = (H * w[y].double()).sum(1)
        assert float((lse.double() - ref_lse).abs().max()) < 1e-4 and float((loss.double() - (ref_lse - target)).abs().max()) < 1e-4
        ref_dh = (ref_dh / total[:, None] - w[y].double()) / T
        # two independent roundings to 16 bits
        assert float((dh.double() - ref_dh).norm()) <= 2 * 2.0 ** -8 * float(ref_dh.norm())
        at = torch.tensor([0, 5, 1048575, 1048576, V - 2, V - 1], device="cuda")
        d = torch.exp(H @ w[at].double().t() - ref_lse[:, None]) - (at[None, :] == y[:, None]).double()
        ref_dw = (d / T).t() @ H
        assert float((dw[at].double() - ref_dw).norm()) <= 2 * 2.0 ** -8 * float(ref_dw.norm())


def test_dropout_past_four_gigabytes():
    import torch
    rows, cols, ld = 70000, 33000, 33008       # 4.6e9 bytes
    x = torch.ones(rows, ld, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    cdl.cdl_dropout(x, ld, None, 0, y, ld, cdl.CDL_BF16, rows, cols, 0.5, 9, 4)
    part = torch.empty(3, cols, dtype=torch.bfloat16, device="cuda")
    for r in (0, 40000, rows - 3):             # the same rows as calls of their own
        cdl.cdl_dropout(x[r:], ld, None, 0, part, cols, cdl.CDL_BF16, 3, cols, 0.5, 9, 4 + r * cols)
        assert torch.equal(part, y[r:r + 3, :cols])


@pytest.mark.parametrize("T,D", [(1, 2 ** 30), (2, 2 ** 30 - 523), (3, 2 ** 30)])
def test_longest_rows_of_the_vocabulary_loss(T, D):
    """Rows at the largest reduced dimension: their bytes pass 31 bits, and a tile's stages take longer than the limit of a single wait."""
    import torch
    V, pitch = 2, -(-D // 8) * 8
    g = torch.Generator().manual_seed(D % 1000 + T)
    at = torch.tensor([0, 1, 2 ** 29 + 7, D - 700, D - 2, D - 1])          # the only entries that are not 0
    h, w = (torch.zeros(n, pitch, dtype=torch.bfloat16, device="cuda") for n in (T, V))
    hv, wv = (torch.randn(n, len(at), generator=g).to(torch.bfloat16) for n in (T, V))
    h[:, at.cuda()], w[:, at.cuda()] = hv.cuda(), wv.cuda()
    y = (torch.arange(T) % V).cuda()
    loss, lse = torch.full((T,), -7.0, device="cuda"), torch.full((T,), -7.0, device="cuda")
    grad = T > 2
    nb = cdl.cdl_vocab_loss_workspace_bytes(T, V, D, grad)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    cdl.cdl_vocab_loss_fwd(h, pitch, w, pitch, cdl.CDL_BF16, y, T, V, D, loss, lse, ws, nb)
    cdl.cdl_workspace_status(ws)
    logits = hv.double() @ wv.double().t()
    ref = torch.logsumexp(logits, 1)
    # six products of normal numbers in binary32, exponentials to 2^-21
    assert float((lse.double().cpu() - ref).abs().max()) < 1e-5
    assert float((loss.double().cpu() - (ref - logits[torch.arange(T), y.cpu()])).abs().max()) < 1e-5
    if not grad:
        return
    gl = torch.full((T,), 1.0 / T, device="cuda")
    dh, dw = torch.full_like(h, 9.0), torch.full_like(w, 9.0)
    cdl.cdl_vocab_loss_bwd(h, pitch, w, pitch, cdl.CDL_BF16, y, lse, gl, T, V, D, dh, pitch, dw, pitch, ws, nb)
    cdl.cdl_workspace_status(ws)
    dl = (torch.exp(logits - ref[:, None]) - (torch.arange(V)[None, :] == y.cpu()[:, None]).double()) / T
    for got, a, b in ((dh, dl, wv.double()), (dw, dl.t(), hv.double())):
        # two roundings to 16 bits (dl and the result)
        assert bool(((got[:, at.cuda()].double().cpu() - a @ b).abs() <= 2 * 2.0 ** -8 * (a.abs() @ b.abs())).all())
        for row in got:
            assert int(torch.count_nonzero(row[:D])) == int(torch.count_nonzero(row[at.cuda()]))
