"""Layer norm at the ends of the numbers' range, in every form of the kernels."""
import pytest

import paper_2501_09849_b200 as cdl

pytestmark = pytest.mark.gpu
TYPES = {"f32": (cdl.CDL_F32, "float32", 2.0 ** -24), "bf16": (cdl.CDL_BF16, "bfloat16", 2.0 ** -8), "f16": (cdl.CDL_F16, "float16", 2.0 ** -11)}
COLS = [1, 100, 128, 257, 300, 1000, 1001, 1500, 3000, 4099, 5000, 9000, 9001, 20000, 40004, 70000, 70001]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_gradient_of_a_row_whose_mean_times_rstd_overflows(kind, cols):
    """Rows of equal large entries, rstd that of eps alone: n is 0 and dx = rstd (a - mean a), where 0 in the place of what a row does not have would
    be -infinity times 0."""
    import torch
    code, dtype, u = TYPES[kind]
    dt, rows = getattr(torch, dtype), 5
    x = torch.full((rows, cols), 2e36, device="cuda").to(dt)
    dy = torch.randn(rows, cols, generator=torch.Generator().manual_seed(cols)).to(dt).cuda()
    gamma = torch.randn(cols, generator=torch.Generator().manual_seed(1)).cuda()
    mean, rstd = x[:, 0].float().contiguous(), torch.full((rows,), 316.0, device="cuda")
    nb = cdl.cdl_layernorm_workspace_bytes(rows, cols)
    ws, dx, dg, db = torch.empty(nb, dtype=torch.uint8, device="cuda"), torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    cdl.cdl_layernorm_bwd(dy, cols, x, cols, code, gamma, mean, rstd, rows, cols, None, 0, dx, cols, dg, db, ws=ws, ws_bytes=nb)
    a = dy.double() * gamma.double()
    ref, size = 316.0 * (a - a.mean(1, True)), 316.0 * (a.abs() + a.abs().mean(1, True))
    # a thread adds at most cols / 512 + 32 terms one after the other, then ten exchanges
    assert bool(((dx.double() - ref).abs() <= ref.abs() * u + size * (cols / 512 + 64) * 2.0 ** -24).all())
    assert bool((dg == 0).all()) and bool(((db.double() - dy.double().sum(0)).abs() <= dy.double().abs().sum(0) * 8 * 2.0 ** -24).all())


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("cols", COLS[1:] + [140001])
def test_statistics_of_a_row_that_is_not_finite(kind, cols):
    """mean and rstd of a row with a NaN or an infinity are NaN, or an infinity the mean, as the row is NaN; the other rows keep theirs."""
    import torch
    code, dtype, _ = TYPES[kind]
    x = torch.randn(6, cols, generator=torch.Generator().manual_seed(2)).to(getattr(torch, dtype)).cuda()
    y, clean = torch.empty_like(x), torch.empty_like(x)
    mean, rstd, m0, r0 = (torch.empty(6, device="cuda") for _ in range(4))
    cdl.cdl_layernorm_fwd(x, cols, code, None, None, 6, cols, 1e-5, clean, cols, m0, r0)
    x[1, cols // 2], x[3, cols - 1], x[4, 0] = float("nan"), float("inf"), float("-inf")
    cdl.cdl_layernorm_fwd(x, cols, code, None, None, 6, cols, 1e-5, y, cols, mean, rstd)
    bad, good = [1, 3, 4], [0, 2, 5]
    assert bool(y[bad].isnan().all()) and bool(rstd[bad].isnan().all()) and not bool(mean[bad].isfinite().any())
    assert torch.equal(y[good], clean[good]) and torch.equal(mean[good], m0[good]) and torch.equal(rstd[good], r0[good])
