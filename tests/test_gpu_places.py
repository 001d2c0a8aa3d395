"""Layer norm and activations with a pitch and an offset of its own for every tensor (some that start on 16 bytes beside some that do not), weights off 16
bytes, several rows a block or cluster, against 64-bit values."""
import math

import pytest

import paper_2501_09849_b200 as cdl
from placed import Placed

pytestmark = pytest.mark.gpu
TYPES = {"f32": (cdl.CDL_F32, "float32", 2.0 ** -24), "bf16": (cdl.CDL_BF16, "bfloat16", 2.0 ** -8), "f16": (cdl.CDL_F16, "float16", 2.0 ** -11)}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}
E24 = 2.0 ** -24
# (pad to a multiple of 8 and more, or any; offset) of x, y, dy, residual, dx; offset of gamma and of beta in floats
PLACES = {"pitches": ([("up", 0), ("up+8", 8), ("up+16", 16), ("up", 8), ("up+24", 0)], 0, 0),
          "weights off 16 bytes": ([("up", 0)] * 5, 1, 2),
          "x off": ([(3, 1), ("up", 0), ("up", 0), ("up+8", 0), ("up", 0)], 0, 3),
          "outputs off": ([("up", 0), (1, 5), ("up", 8), ("up", 0), (6, 2)], 2, 0),
          "each its own": ([(1, 1), (2, 2), (0, 3), (5, 4), (7, 7)], 3, 1)}


def put(torch, rows, cols, kind, place, fill=None):
    pad, offset = place
    if isinstance(pad, str):
        pad = -cols % 8 + int(pad[3:] or 0)
    return Placed(torch, rows, cols, getattr(torch, TYPES[kind][1]), pad, offset, fill)


def normal(torch, shape, seed, mean=0.0):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") + mean


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("place", list(PLACES))
@pytest.mark.parametrize("rows,cols", [(1, 77), (70, 257), (900, 300), (29, 1000), (700, 1501), (450, 4095), (60, 5000), (170, 9001), (150, 16400), (60, 33000), (3, 70001), (2, 140004)])
def test_layer_norm(kind, place, rows, cols):
    import torch
    code, _, u = TYPES[kind]
    (px, py, pd, pr, pdx), at_g, at_b = PLACES[place]
    x, dy, r = (put(torch, rows, cols, kind, p, normal(torch, (rows, cols), i, m)) for p, i, m in ((px, 1, 0.7), (pd, 2, 0.0), (pr, 3, 0.0)))
    y, dx = put(torch, rows, cols, kind, py), put(torch, rows, cols, kind, pdx)
    gamma, beta = (torch.empty(cols + 4, device="cuda")[at:at + cols] for at in (at_g, at_b))
    gamma.copy_(normal(torch, (cols,), 4, 1.0))
    beta.copy_(normal(torch, (cols,), 5))
    mean, rstd = torch.empty(rows + 1, device="cuda")[1:], torch.empty(rows, device="cuda")
    cdl.cdl_layernorm_fwd(x, x.ld, code, gamma, beta, rows, cols, 1e-5, y, y.ld, mean, rstd)
    # a thread adds at most cols / 512 + 32 terms of a row one after the other, then ten exchanges; the statistics' few roundings
    k = (cols / 512 + 64) * E24
    xd, gd, bd = x.values.double(), gamma.double(), beta.double()
    m = xd.mean(1, True)
    s = ((xd - m) ** 2).mean(1, True).add(1e-5).rsqrt()
    n = (xd - m) * s
    ref = n * gd + bd
    assert bool(((mean.double() - m[:, 0]).abs() <= 2 * E24 * m[:, 0].abs() + k / s[:, 0]).all()) and bool(((rstd.double() - s[:, 0]).abs() <= k * s[:, 0]).all())
    assert bool(((y.values.double() - ref).abs() <= ref.abs() * u + k * (n.abs() + 1) * gd.abs() + 2 * E24 * ((n * gd).abs() + bd.abs())).all())
    nb = cdl.cdl_layernorm_workspace_bytes(rows, cols)
    ws, dg, db = torch.full((nb + 64,), 171, dtype=torch.uint8, device="cuda"), torch.empty(cols + 1, device="cuda")[1:], torch.empty(cols, device="cuda")
    cdl.cdl_layernorm_bwd(dy, dy.ld, x, x.ld, code, gamma, mean, rstd, rows, cols, r, r.ld, dx, dx.ld, dg, db, ws=ws, ws_bytes=nb)
    md, sd = mean.double()[:, None], rstd.double()[:, None]
    n, dyd = (xd - md) * sd, dy.values.double()
    a = dyd * gd
    ref = sd * (a - a.mean(1, True) - n * (a * n).mean(1, True)) + r.values.double()
    bound = sd * (a.abs() + a.abs().mean(1, True) + n.abs() * (a * n).abs().mean(1, True))
    assert bool(((dx.values.double() - ref).abs() <= ref.abs() * u + k * bound + 2 * E24 * ref.abs() + 2 * E24 * (md.abs() * sd) * bound).all())
    krows = (rows / 8 + 100) * E24
    assert bool(((dg.double() - (dyd * n).sum(0)).abs() <= krows * (dyd * n).abs().sum(0) + 4 * E24 * ((md.abs() * sd) * dyd.abs()).sum(0)).all())
    assert bool(((db.double() - dyd.sum(0)).abs() <= krows * dyd.abs().sum(0)).all())
    assert all(t.guarded() for t in (x, y, dy, r, dx)) and bool((ws[nb:] == 171).all())


@pytest.mark.parametrize("cols", [100, 997, 2500, 9003])
def test_far_off_rows_whose_pitch_is_padded(cols):
    """Rows that start on 16 bytes and end inside a unit, mean times rstd beyond binary32 (other widths: the tests of the norm's limits)."""
    import torch
    rows = 5
    x = put(torch, rows, cols, "bf16", ("up", 0), torch.full((rows, cols), 2e36, device="cuda"))
    dy = put(torch, rows, cols, "bf16", ("up+8", 8), normal(torch, (rows, cols), 1))
    dx, mean, rstd = put(torch, rows, cols, "bf16", ("up", 0)), x.values[:, 0].float().contiguous(), torch.full((rows,), 316.0, device="cuda")
    cdl.cdl_layernorm_bwd(dy, dy.ld, x, x.ld, cdl.CDL_BF16, None, mean, rstd, rows, cols, None, 0, dx, dx.ld)
    d = dy.values.double()
    ref, size = 316.0 * (d - d.mean(1, True)), 316.0 * (d.abs() + d.abs().mean(1, True))
    assert bool(((dx.values.double() - ref).abs() <= ref.abs() * 2.0 ** -8 + size * (cols / 512 + 64) * E24).all()) and dx.guarded()


def gelu(torch, z):
    p = 0.5 * torch.erfc(-z * math.sqrt(0.5))
    return z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("place", list(PLACES))
@pytest.mark.parametrize("rows,cols", [(1, 77), (9, 128), (17, 1023), (130, 1111), (33, 2056), (5, 9000)])
def test_activation(kind, place, rows, cols):
    import torch
    code, _, u = TYPES[kind]
    px, py, pd, pa, pdx = PLACES[place][0]
    x, dy = put(torch, rows, cols, kind, px, 2 * normal(torch, (rows, cols), 1)), put(torch, rows, cols, kind, pd, normal(torch, (rows, cols), 2))
    y, again, dx = (put(torch, rows, cols, kind, p) for p in (py, pa, pdx))
    ldc, groups = -(-cols // 16) * 16 + 32, -(-cols // 128)
    codes, scales = torch.full((rows, ldc), 77, dtype=torch.uint8, device="cuda"), torch.empty(groups, rows, device="cuda")
    cdl.cdl_act_fwd(x, x.ld, code, cdl.CDL_ACT_GELU, rows, cols, y, y.ld, codes, ldc, scales)
    plain, ref_c, ref_s = x.values.float().contiguous(), torch.zeros_like(codes), torch.empty_like(scales)
    cdl.cdl_fp8_quantize(plain, cols, cdl.CDL_F32, rows, cols, cdl.CDL_FP8_ROWS, ref_c, ldc, ref_s)
    assert torch.equal(codes[:, :cols], ref_c[:, :cols]) and torch.equal(scales, ref_s) and bool((codes[:, cols:] == 77).all())
    v, _ = gelu(torch, x.values.double())

    def slack(z):       # the exponential's argument is rounded twice: 2 z^2 roundings of it, and some sixteen others
        return (16 + 2 * z.abs().clamp(max=14.5) ** 2) * E24
    assert bool(((y.values.double() - v).abs() <= v.abs() * (u + slack(x.values.double())) + TINY[kind]).all())
    cdl.cdl_act_bwd(dy, dy.ld, codes, ldc, scales, code, cdl.CDL_ACT_GELU, rows, cols, dx, dx.ld, again, again.ld)
    z = codes[:, :cols].contiguous().view(torch.float8_e4m3fn).double() * scales.double().t().repeat_interleave(128, 1)[:, :cols]
    v, s = gelu(torch, z)
    want, d = dy.values.double() * s, dy.values.double().abs()
    assert bool(((dx.values.double() - want).abs() <= want.abs() * u + d * (1 + z.abs()) * (2 * slack(z) + 4 * E24) + TINY[kind]).all())
    assert bool(((again.values.double() - v).abs() <= v.abs() * (u + 1.5 * slack(z) + 2.0 ** -22) + TINY[kind]).all())
    assert all(t.guarded() for t in (x, y, dy, again, dx))
