"""Linear layers in every form that a plan can choose, each with more reduced entries than one segment holds and the whole epilogue: whole tiles of CTA
pairs and of single CTAs, those with runs of stages behind them, clusters, few rows; outputs that leave by TMA and such that do not; a pitch and an offset
of its own for every tensor.  What form a size has is asserted."""
import math

import pytest

import paper_2501_09849_b200 as cdl
from linear_plan import forward_form, tile_plan
from placed import Placed

pytestmark = pytest.mark.gpu
TYPES = {"f32": (cdl.CDL_F32, "float32", 2.0 ** -24), "bf16": (cdl.CDL_BF16, "bfloat16", 2.0 ** -8), "f16": (cdl.CDL_F16, "float16", 2.0 ** -11)}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}


def up(n, m):
    return -(-n // m) * m


def operand(torch, rows, cols, kind, std, seed, extra=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    m = torch.full((rows, up(cols, 8) + extra), float("nan"), dtype=getattr(torch, TYPES[kind][1]), device="cuda")
    m[:, :cols] = (torch.randn(rows, cols, generator=g, device="cuda") * std).to(m.dtype)
    return m


def normal(torch, shape, seed, std=1.0):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * std


def slack(R, out):
    # An instruction of 16 reduced entries cuts what it adds to by at most 2^-23 of the magnitudes so far, in a segment of n instructions n / 2 times that of
    # the segment's; segments, pieces (148 at most, each added to once) and the bias are rounded.
    segment = 512 if out == "f32" else 1024
    return (min(R, segment) / 16 / 2 + 1) * 2.0 ** -23 + (R / segment + 148 / 16 + 4) * 2.0 ** -24


def gelu(torch, z):
    p = 0.5 * torch.erfc(-z * math.sqrt(0.5))
    return z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


# output, (pad, offset) of the output, of the residual; a binary32 bias' offset
PLACES = [("f32", (0, 0), (0, 0), 0), ("f32", (4, 0), (3, 1), 1), ("bf16", (0, 0), (8, 8), 2), ("bf16", (8, 0), (0, 1), 0), ("f16", (5, 3), (16, 8), 3)]
FORWARD = [(5, 1003, 3000, "rows"), (100, 301, 5000, "cluster"), (300, 300, 20000, "singles with runs"), (1031, 2003, 1090, "singles"), (2203, 2301, 1700, "pairs"),
           (2300, 2305, 5000, "pairs with runs"), (4100, 3001, 1090, "pairs")]


@pytest.mark.parametrize("out,place,res_place,bias_at", PLACES)
@pytest.mark.parametrize("M,N,K,form", FORWARD)
def test_forward(M, N, K, form, out, place, res_place, bias_at):
    import torch
    assert forward_form(M, N, K) == form
    kind = "f16" if out == "f16" else "bf16"
    ocode, dtype, u = TYPES[out]
    N -= N % 8 if place == (0, 0) else 0                 # (rows of 16 bytes, once for every size)
    a, w = operand(torch, M, K, kind, 1.0, 1), operand(torch, N, K, kind, 1 / math.sqrt(K), 2, 8)
    bias = torch.empty(N + 8, device="cuda")[bias_at:bias_at + N]
    bias.copy_(normal(torch, (N,), 3, 0.3))
    r = Placed(torch, M, N, getattr(torch, dtype), *res_place, fill=normal(torch, (M, N), 4))
    nb, ldc, groups = cdl.cdl_linear_workspace_bytes(M, N, K), up(N, 16) + 16, -(-N // 128)
    ws = torch.full((nb + 64,), 171, dtype=torch.uint8, device="cuda")
    z = a[:, :K].double() @ w[:, :K].double().t() + bias.double()
    size = a[:, :K].double().abs() @ w[:, :K].double().abs().t() + bias.double().abs()
    tz = size * slack(K, out)
    v = gelu(torch, z)[0]
    ref = v + r.values.double()
    # (GELU's slope is at most 1.13, its own error below 2^-18 of z)
    tol = 1.2 * tz + z.abs() * 2.0 ** -18 + ref.abs() * (u + 2.0 ** -23) + TINY[out]
    results = []
    for keep in (True, False):
        o = Placed(torch, M, N, getattr(torch, dtype), *place)
        codes, scales = torch.full((M, ldc), 77, dtype=torch.uint8, device="cuda"), torch.full((groups, M), -1.0, device="cuda")
        cdl.cdl_linear_fwd(a, a.stride(0), w, w.stride(0), TYPES[kind][0], bias, cdl.CDL_ACT_GELU, r, r.ld, M, N, K, o, o.ld, ocode, codes if keep else None, ldc if keep else 0,
                           scales if keep else None, ws=ws, ws_bytes=nb)
        cdl.cdl_workspace_status(ws)
        assert o.guarded() and r.guarded() and bool((ws[nb:] == 171).all())
        err = (o.values.double() - ref).abs()
        assert bool((err <= tol).all()), float((err / tol).max())
        results.append(o.values.clone())
        if keep:
            zs = scales.double().t().repeat_interleave(128, 1)[:, :N]
            kept = codes[:, :N].contiguous().view(torch.float8_e4m3fn).double() * zs
            assert bool(((kept - z).abs() <= torch.maximum(z.abs() * 2.0 ** -4, zs * 2.0 ** -10) * (1 + 2.0 ** -18) + 1.1 * tz).all())
            largest, tl = (torch.nn.functional.pad(t, (0, groups * 128 - N)).view(M, groups, 128).amax(2).t() / 448 for t in (z.abs(), tz))
            assert bool(((scales.double() - largest).abs() <= largest * 2.0 ** -22 + tl).all())
            assert bool((codes[:, N:] == 77).all())
    assert torch.equal(*results)
    cdl.cdl_linear_fwd(a, a.stride(0), w, w.stride(0), TYPES[kind][0], bias, cdl.CDL_ACT_GELU, r, r.ld, M, N, K, r, r.ld, ocode, ws=ws, ws_bytes=nb)       # over the residual
    assert torch.equal(r.values, results[0]) and r.guarded()


DATA = [(7, 3000, 1003, "cluster"), (100, 5000, 301, "cluster"), (300, 20000, 300, "singles with runs"), (1031, 1090, 2003, "singles"), (2203, 1700, 2301, "pairs"),
        (2300, 5000, 2305, "pairs with runs"), (4100, 600, 3001, "pairs")]


@pytest.mark.parametrize("out,place,res_place,bias_at", PLACES)
@pytest.mark.parametrize("M,N,K,form", DATA)
def test_data_gradient(M, N, K, form, out, place, res_place, bias_at):
    import torch
    assert tile_plan(M, K, N).form == form
    kind = "f16" if out == "f16" else "bf16"
    ocode, dtype, u = TYPES[out]
    K -= K % 8 if place == (0, 0) else 0
    dy, w = operand(torch, M, N, kind, 1.0, 1), operand(torch, N, K, kind, 1 / math.sqrt(N), 2, 8)
    r = Placed(torch, M, K, getattr(torch, dtype), *res_place, fill=normal(torch, (M, K), 4))
    nb, ldc, groups = cdl.cdl_linear_workspace_bytes(M, N, K), up(K, 16) + 16, -(-K // 128)
    ws = torch.full((nb + 64,), 171, dtype=torch.uint8, device="cuda")
    codes, scales = torch.full((M, ldc), 127, dtype=torch.uint8, device="cuda"), torch.empty(groups, M, device="cuda")       # (NaN between the rows)
    z = normal(torch, (M, K), 5, 1.2)
    cdl.cdl_fp8_quantize(z, K, cdl.CDL_F32, M, K, cdl.CDL_FP8_ROWS, codes, ldc, scales)
    z8 = codes[:, :K].contiguous().view(torch.float8_e4m3fn).double() * scales.double().t().repeat_interleave(128, 1)[:, :K]
    core, size = dy[:, :N].double() @ w[:, :K].double(), dy[:, :N].double().abs() @ w[:, :K].double().abs() * slack(N, out)
    for act, res in ((cdl.CDL_ACT_GELU, True), (cdl.CDL_ACT_GELU, False), (cdl.CDL_ACT_NONE, True)):
        o = Placed(torch, M, K, getattr(torch, dtype), *place)
        kept = act != cdl.CDL_ACT_NONE
        cdl.cdl_linear_bwd_data(dy, dy.stride(0), w, w.stride(0), TYPES[kind][0], act, codes if kept else None, ldc if kept else 0, scales if kept else None, r if res else None, r.ld,
                                M, N, K, o, o.ld, ocode, ws=ws, ws_bytes=nb)
        cdl.cdl_workspace_status(ws)
        ref = core * gelu(torch, z8)[1] if kept else core
        ref = ref + r.values.double() if res else ref
        tol = 1.2 * size + core.abs() * 2.0 ** -17 + ref.abs() * (u + 2.0 ** -23) + TINY[out]
        err = (o.values.double() - ref).abs()
        assert bool((err <= tol).all()), float((err / tol).max())
        assert o.guarded() and r.guarded() and bool((ws[nb:] == 171).all())


WEIGHT = [(8192, 512, 256, "cluster"), (5000, 100, 301, "cluster"), (50000, 130, 72, "singles with runs"), (1090, 1031, 2003, "singles"), (1700, 2203, 2301, "pairs"),
          (6000, 2304, 2305, "pairs with runs"), (600, 4100, 3001, "pairs")]


@pytest.mark.parametrize("out,place", [p[:2] for p in PLACES])
@pytest.mark.parametrize("M,N,K,form", WEIGHT)
def test_weight_gradient(M, N, K, form, out, place):
    import torch
    assert tile_plan(N, K, M).form == form
    kind = "f16" if out == "f16" else "bf16"
    ocode, dtype, u = TYPES[out]
    K -= K % 8 if place == (0, 0) else 0
    dy, a = operand(torch, M, N, kind, 1.0, 1), operand(torch, M, K, kind, 0.1, 2, 8)
    nb = cdl.cdl_linear_workspace_bytes(M, N, K)
    ws = torch.full((nb + 64,), 171, dtype=torch.uint8, device="cuda")
    core, size = dy[:, :N].double().t() @ a[:, :K].double(), dy[:, :N].double().abs().t() @ a[:, :K].double().abs() * slack(M, out)
    before = normal(torch, (N, K), 4)
    for accumulate in (False, True):
        o, db = Placed(torch, N, K, getattr(torch, dtype), *place, fill=before), torch.full((N,), 7.0, device="cuda")
        ref = core + o.values.double() if accumulate else core
        cdl.cdl_linear_bwd_weight(dy, dy.stride(0), a, a.stride(0), TYPES[kind][0], M, N, K, accumulate, o, o.ld, ocode, db, ws=ws, ws_bytes=nb)
        cdl.cdl_workspace_status(ws)
        tol = size + ref.abs() * (u + 2.0 ** -23) + TINY[out]
        err = (o.values.double() - ref).abs()
        assert bool((err <= tol).all()), float((err / tol).max())
        assert o.guarded() and bool((ws[nb:] == 171).all())
        assert bool(((db.double() - dy[:, :N].double().sum(0)).abs() <= dy[:, :N].double().abs().sum(0) * (M / 256 + 60) * 2.0 ** -24).all())
