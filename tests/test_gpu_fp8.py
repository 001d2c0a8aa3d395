"""Block-scaled 8-bit floating point: the quantizer bit for bit against its definition, its error in 64 bits, and the
product against 64-bit sums."""
import pytest

import paper_2501_09849_b200 as cdl

pytestmark = pytest.mark.gpu

TYPES = {"f32": (cdl.CDL_F32, "float32", 2.0 ** -24), "bf16": (cdl.CDL_BF16, "bfloat16", 2.0 ** -8), "f16": (cdl.CDL_F16, "float16", 2.0 ** -11)}
MODES = {"rows": cdl.CDL_FP8_ROWS, "blocks": cdl.CDL_FP8_BLOCKS}


def up(n, m=16):
    return -(-n // m) * m


def plain_quantize(torch, x, mode):
    """The definition, in binary32 on the host; x: rows x cols floats."""
    rows, cols = x.shape
    size = 1 if mode == "rows" else 128
    pad = torch.zeros(up(rows, size), up(cols, 128))
    pad[:rows, :cols] = x
    b = pad.view(up(rows, size) // size, size, -1, 128)
    a = b.abs()
    amax = torch.where(a.isnan(), torch.zeros_like(a), a).amax(dim=(1, 3))
    s = torch.clamp(amax * (torch.ones(()) / 448.0), min=2.0 ** -126)
    v = b * (1.0 / s)[:, None, :, None]
    codes = v.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return codes.view(pad.shape)[:rows, :cols].contiguous(), s.t().contiguous()


def same_codes(torch, a, b):
    """Equal bytes, except that either sign of NaN is the NaN code."""
    a, b = a.contiguous().view(torch.uint8).cpu(), b.contiguous().view(torch.uint8).cpu()
    return bool(((a == b) | (((a & 127) == 127) & ((b & 127) == 127))).all())


def run_quantize(torch, x, kind, mode, both, ldx=None):
    rows, cols = x.shape
    ldx = x.stride(0) if ldx is None else ldx
    f8 = torch.float8_e4m3fn
    codes = torch.full((rows, up(cols) + 16), 3.0, device="cuda").to(f8)
    groups = rows if mode == "rows" else -(-rows // 128)
    groups_t = cols if mode == "rows" else -(-cols // 128)
    scales = torch.full((-(-cols // 128), groups), -1.0, device="cuda")
    ct = torch.full((cols, up(rows) + 32), 3.0, device="cuda").to(f8) if both else None
    st = torch.full((-(-rows // 128), groups_t), -1.0, device="cuda") if both else None
    cdl.cdl_fp8_quantize(x, ldx, TYPES[kind][0], rows, cols, MODES[mode], codes, codes.stride(0), scales, ct, ct.stride(0) if both else 0, st)
    assert bool((codes[:, cols:].float() == 3.0).all())
    if both:
        assert bool((ct[:, rows:].float() == 3.0).all())
        return codes[:, :cols], scales, ct[:, :rows], st
    return codes[:, :cols], scales, None, None


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("rows,cols,pad,offset", [(1, 1, 0, 0), (1, 128, 0, 0), (1, 1000, 0, 0), (3, 129, 7, 0), (128, 128, 0, 0), (129, 255, 1, 1),
                                                  (200, 640, 16, 8), (517, 333, 0, 0), (1000, 72, 0, 0)])
def test_quantizer_is_its_definition(kind, mode, rows, cols, pad, offset):
    import torch
    dt = getattr(torch, TYPES[kind][1])
    g = torch.Generator().manual_seed(rows * 1000 + cols)
    flat = torch.randn(offset + rows * (cols + pad) + 16, generator=g) * torch.exp(2 * torch.randn(offset + rows * (cols + pad) + 16, generator=g))
    flat = flat.to(dt).cuda()
    x = flat[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    codes, scales, ct, st = run_quantize(torch, x, kind, mode, True)
    only, only_s, _, _ = run_quantize(torch, x, kind, mode, False)
    xh = x.float().cpu()
    ref, ref_s = plain_quantize(torch, xh, mode)
    assert torch.equal(scales.cpu(), ref_s) and same_codes(torch, codes, ref)
    assert torch.equal(only_s, scales) and same_codes(torch, only, codes)
    ref, ref_s = plain_quantize(torch, xh.t().contiguous(), mode)
    assert torch.equal(st.cpu(), ref_s) and same_codes(torch, ct, ref)
    # in 64 bits: an entry is off by at most half a step of its code: 2^-4 of the value, or 2^-10 scales below the smallest
    # normal code; two roundings of binary32 (the reciprocal and the product) come before the code's own
    s = scales.double().cpu()
    s = s if mode == "rows" else s.repeat_interleave(128, 1)[:, :rows]
    s = s.t().repeat_interleave(128, 1)[:, :cols]
    err = (codes.double().cpu() * s - xh.double()).abs()
    assert bool((err <= torch.maximum(xh.double().abs() * 2.0 ** -4, s * 2.0 ** -10) * (1 + 2.0 ** -18)).all())


@pytest.mark.parametrize("mode", list(MODES))
def test_quantizer_zero_tiny_huge_and_non_finite_groups(mode):
    import torch
    x = torch.zeros(384, 384)
    x[0:128, 128:256] = 1e-44                     # subnormal: the smallest scale
    x[0:128, 256:384] = 3e38
    x[200, 5] = float("nan")                      # no part of the scale
    x[201, 6] = 2.0
    x[300, 130] = float("inf")                    # its group is lost, the others are not
    x[301, 131] = -4.0
    codes, scales, ct, st = run_quantize(torch, x.cuda(), "f32", mode, True)
    ref, ref_s = plain_quantize(torch, x, mode)
    assert torch.equal(scales.cpu(), ref_s) and same_codes(torch, codes, ref)
    assert float(scales[0, 0]) == 2.0 ** -126
    ref, ref_s = plain_quantize(torch, x.t().contiguous(), mode)
    assert torch.equal(st.cpu(), ref_s) and same_codes(torch, ct, ref)
    assert cdl.cdl_fp8_quantize(None, 0, cdl.CDL_F32, 0, 7, MODES[mode], None, 0, None) == 0


def operand(torch, rows, cols, mode, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    codes = torch.zeros(rows, up(cols)).to(torch.float8_e4m3fn)
    codes[:, :cols] = (torch.randn(rows, cols, generator=g) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
    codes[:, cols:] = torch.full((rows, up(cols) - cols), float("nan")).to(torch.float8_e4m3fn)       # the pitch's padding is not read
    groups = rows if mode == "rows" else -(-rows // 128)
    scales = torch.exp(torch.randn(-(-cols // 128), groups, generator=g) * spread) * 1e-2
    return codes, scales


def values(codes, scales, rows, cols, mode):
    s = scales.double()
    s = s if mode == "rows" else s.repeat_interleave(128, 1)[:, :rows]
    return codes[:, :cols].double() * s.t().repeat_interleave(128, 1)[:, :cols]


def run_matmul(torch, M, N, K, mode, out, bias=None, pad=0, seed=0, offset=0, stream=None):
    a, sa = operand(torch, M, K, "rows", seed + 1)
    b, sb = operand(torch, N, K, mode, seed + 2)
    code, dtype, u = TYPES[out]
    flat = torch.full((offset + M * (N + pad),), 5.0, dtype=getattr(torch, dtype), device="cuda")
    o = flat[offset:].view(M, N + pad)
    nb = cdl.cdl_fp8_matmul_workspace_bytes(M, N, K)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    ag, sag, bg, sbg = a.cuda(), sa.cuda(), b.cuda(), sb.cuda()
    cdl.cdl_fp8_matmul(ag, ag.stride(0), sag, bg, bg.stride(0), sbg, MODES[mode], M, N, K, o, N + pad, code,
                       None if bias is None else bias.cuda(), ws, nb, stream=stream)
    cdl.cdl_workspace_status(ws)
    assert bool((o[:, N:] == 5.0).all()) and bool((flat[:offset] == 5.0).all())
    A, B = values(a.cuda(), sa.cuda(), M, K, "rows"), values(b.cuda(), sb.cuda(), N, K, mode)
    ref, size = A @ B.t(), A.abs() @ B.abs().t()
    if bias is not None:
        ref, size = ref + bias.double().cuda(), size + bias.abs().double().cuda()
    # per block of 128: four tensor-core sums, each good to 2^-22 of its terms' magnitudes; the product of the two scales and
    # one fused multiply-add per block in binary32; the cluster's sums (at most 8) and the bias; the rounding to the type
    kb = -(-K // 128)
    tol = size * (4 * 2.0 ** -22 + (kb + 12) * 2.0 ** -24) + ref.abs() * u
    err = (o[:, :N].double() - ref).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
    return o[:, :N]


@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("M,N,K,pad,offset,out", [
    (1, 1, 1, 0, 0, "f32"), (1, 4096, 4096, 0, 0, "bf16"), (1, 100, 10000, 0, 0, "f16"), (2, 128, 128, 0, 0, "f32"), (7, 129, 257, 3, 0, "f32"),
    (33, 1000, 1111, 0, 1, "bf16"), (64, 512, 2048, 8, 0, "f16"), (128, 256, 384, 0, 0, "f32"), (129, 300, 640, 0, 0, "bf16"),
    (1009, 2304, 1000, 0, 0, "f16"), (300, 4000, 272, 0, 0, "f32"), (2304, 2304, 512, 0, 0, "f32"), (2300, 2310, 640, 2, 0, "bf16"),
    (2561, 2001, 144, 0, 1, "f16"), (4000, 1500, 129, 0, 0, "f32"), (3001, 5003, 130, 0, 0, "bf16"),
    (2304, 2304, 9000, 0, 0, "f32"), (2301, 2303, 8300, 1, 0, "bf16"), (4800, 1100, 6200, 0, 0, "f16"),      # the last round's tiles in parts
])
def test_product(mode, M, N, K, pad, offset, out):
    import torch
    run_matmul(torch, M, N, K, mode, out, pad=pad, seed=M + N + K, offset=offset)


@pytest.mark.parametrize("M,N,K", [(1, 300, 1024), (2, 77, 513), (200, 300, 256), (2500, 2500, 256), (2304, 2304, 8192)])
def test_product_with_bias(M, N, K):
    import torch
    bias = torch.randn(N, generator=torch.Generator().manual_seed(3)) * 3
    for out in TYPES:
        run_matmul(torch, M, N, K, "blocks", out, bias=bias, seed=5)


# Few tiles and a long reduced dimension: the tiles' stages are one sequence, cut wherever the runs end.  An entry's sum has at
# most as many roundings as there are blocks and pieces, and a piece is at least four blocks but for a tile's first and last.
@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("M,N,K,pad,offset,out", [
    (3, 100, 30000, 3, 0, "f32"), (140, 250, 20001, 0, 1, "bf16"), (12, 3720, 9000, 0, 0, "f16"), (257, 1300, 9000, 1, 0, "f16"),
    (400, 2500, 12300, 0, 0, "bf16"), (1540, 3974, 5000, 2, 0, "f32"), (2301, 2303, 2500, 0, 0, "f32"), (48, 139, 34086, 0, 0, "bf16"),
])
def test_product_in_runs(mode, M, N, K, pad, offset, out):
    import torch
    bias = torch.randn(N, generator=torch.Generator().manual_seed(M)) * 3 if M % 2 == 0 else None
    a = run_matmul(torch, M, N, K, mode, out, bias=bias, pad=pad, seed=M + N + K, offset=offset)
    b = run_matmul(torch, M, N, K, mode, out, bias=bias, pad=pad, seed=M + N + K, offset=offset)
    assert torch.equal(a, b)


# One to four rows, whose products a warp does for eight rows of B at a time: ends of the reduced dimension in every 16-byte unit of a
# block, slices, several passes of a warp.  (A block of 128 is two chains of two matrix instructions: within the four sums
# that the tolerance has.)
@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("M", [1, 2, 3, 4])
@pytest.mark.parametrize("N,K,pad,offset,out", [(9, 16, 0, 0, "f32"), (131, 531, 1, 0, "bf16"), (8, 1024, 0, 0, "f16"), (1000, 113, 0, 1, "f32"), (77, 9999, 0, 0, "f32"),
                                                (4099, 640, 2, 0, "bf16"), (20000, 257, 0, 0, "f16")])
def test_few_rows(mode, M, N, K, pad, offset, out):
    import torch
    bias = torch.randn(N, generator=torch.Generator().manual_seed(M)) * 3 if N % 2 else None
    run_matmul(torch, M, N, K, mode, out, bias=bias, pad=pad, seed=M + N + K, offset=offset)


@pytest.mark.parametrize("M", [1, 4, 7])
def test_codes_that_are_no_numbers_stay_in_their_rows(M):
    import torch
    N, K = 50, 400
    a, sa = operand(torch, M, K, "rows", 1)
    b, sb = operand(torch, N, K, "blocks", 2)
    b[13, 390] = torch.tensor(float("nan")).to(torch.float8_e4m3fn)
    if M > 1:
        a[M - 1, 5] = torch.tensor(float("nan")).to(torch.float8_e4m3fn)
    out = torch.zeros(M, N, device="cuda")
    ws = torch.empty(cdl.cdl_fp8_matmul_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
    cdl.cdl_fp8_matmul(a.cuda(), a.stride(0), sa.cuda(), b.cuda(), b.stride(0), sb.cuda(), MODES["blocks"], M, N, K, out, N, cdl.CDL_F32, None, ws, ws.numel())
    want = torch.zeros(M, N, dtype=torch.bool)
    want[:, 13] = True
    if M > 1:
        want[M - 1] = True
    assert torch.equal(out.cpu().isnan(), want)


def test_product_repeats_and_other_stream():
    import torch
    for M, N, K in ((3, 1000, 4096), (2500, 2400, 640)):
        a = run_matmul(torch, M, N, K, "rows", "f32", seed=9)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            b = run_matmul(torch, M, N, K, "rows", "f32", seed=9)
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(a, b)


def test_product_empty():
    import torch
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    out = torch.full((3, 8), 4.0, device="cuda")
    bias = torch.arange(5, device="cuda", dtype=torch.float32)
    cdl.cdl_fp8_matmul(None, 0, None, None, 0, None, cdl.CDL_FP8_BLOCKS, 3, 5, 0, out, 8, cdl.CDL_F32, bias, ws, 256)
    assert bool((out[:, :5] == bias).all()) and bool((out[:, 5:] == 4.0).all())
    cdl.cdl_fp8_matmul(None, 0, None, None, 0, None, cdl.CDL_FP8_BLOCKS, 3, 5, 0, out, 8, cdl.CDL_F32, None, ws, 256)
    assert bool((out[:, :5] == 0).all())
    assert cdl.cdl_fp8_matmul(None, 0, None, None, 0, None, cdl.CDL_FP8_BLOCKS, 0, 5, 7, None, 8, cdl.CDL_F32, None, ws, 256) == 0


def test_layer_gradients_from_one_quantization_each():
    """Forward, data gradient and weight gradient of Y = X W^T with every operand quantized once (both orientations)."""
    import torch
    T, I, O = 300, 260, 390
    g = torch.Generator().manual_seed(11)
    x = torch.randn(T, I, generator=g).to(torch.bfloat16).cuda()
    w = (torch.randn(O, I, generator=g) / 16).cuda()
    dy = torch.randn(T, O, generator=g).to(torch.bfloat16).cuda()
    xc, xs, xct, xst = run_quantize(torch, x, "bf16", "rows", True)
    wc, wsc, wct, wst = run_quantize(torch, w, "f32", "blocks", True)
    gc, gs, gct, gst = run_quantize(torch, dy, "bf16", "rows", True)
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")

    def product(a, sa, b, sb, mode, M, N, K):
        out = torch.empty(M, N, device="cuda")
        cdl.cdl_fp8_matmul(a, a.stride(0), sa, b, b.stride(0), sb, MODES[mode], M, N, K, out, N, cdl.CDL_F32, None, ws, 256)
        cdl.cdl_workspace_status(ws)
        ref = values(a, sa, M, K, "rows") @ values(b, sb, N, K, mode).t()
        assert float((out - ref).abs().max()) <= 1e-5 * float(ref.abs().max())
        return out.double()

    y = product(xc, xs, wc, wsc, "blocks", T, O, I)
    dx = product(gc, gs, wct, wst, "blocks", T, I, O)
    dw = product(gct, gst, xct, xst, "rows", O, I, T)
    # against the unquantized products: entries are rounded to 2^-4 at most, independently, on both sides
    X, W, G = x.double(), w.double(), dy.double()
    for got, ref in ((y, X @ W.t()), (dx, G @ W), (dw, G.t() @ X)):
        assert float((got - ref).norm() / ref.norm()) < 2 * 2.0 ** -4
