"""Counter-based dropout against a plain implementation: the mask from the generator's definition in 64-bit integers
(numpy), the values in 64-bit floating point."""
import numpy as np
import pytest

import paper_2501_09849_b200 as cdl

pytestmark = pytest.mark.gpu

TYPES = {"f32": (cdl.CDL_F32, "float32"), "bf16": (cdl.CDL_BF16, "bfloat16"), "f16": (cdl.CDL_F16, "float16")}


def words(first, n, seed):
    """Philox4x32-10 words of elements first .. first + n - 1: counter (e div 4, 0), word e mod 4."""
    m, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    lo, hi = first // 4, (first + n + 3) // 4
    b = np.arange(hi - lo, dtype=np.uint64) + np.uint64(lo)
    c = [b & m, b >> sh, np.zeros_like(b), np.zeros_like(b)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> sh) ^ c[1] ^ np.uint64(k[0]), q & m, (p >> sh) ^ c[3] ^ np.uint64(k[1]), p & m]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, 1).reshape(-1)[first - 4 * lo:][:n]


def kept(first, rows, cols, seed, p):
    u = (words(first, rows * cols, seed) >> np.uint64(8)).astype(np.float64) * 2.0 ** -24
    return (u >= float(np.float32(p))).reshape(rows, cols)


def matrix(torch, rows, cols, ld, dtype, seed, offset=0):
    g = torch.Generator().manual_seed(seed)
    flat = torch.randn(offset + rows * ld + 64, generator=g).to(getattr(torch, dtype)).cuda()
    return flat[offset:offset + rows * ld].view(rows, ld)[:, :cols]


def check(torch, y, x, r, mask, p):
    """The very bits: the kept value times the binary32 scale, plus the residual, in one binary32 rounding, then the type's."""
    scale = float(np.float32(1.0 / (1.0 - float(np.float32(p)))))
    xd = x.double().cpu().numpy()
    ref = np.where(mask, xd, 0.0) * scale + (r.double().cpu().numpy() if r is not None else 0.0)
    ref = torch.from_numpy(ref.astype(np.float32)).to(x.dtype)
    assert torch.equal(y.cpu(), ref)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,cols,pad,first,offset", [
    (1, 1, 0, 0, 0), (1, 7, 0, 0, 0), (1, 4096, 0, 4, 0), (3, 8, 8, 0, 0), (5, 24, 40, 12, 0), (37, 129, 0, 0, 0), (37, 129, 3, 2, 0),
    (300, 264, 0, 0, 1), (2, 65, 7, 2 ** 40 + 3, 1), (129, 512, 16, 2 ** 34, 8), (70000, 8, 8, 0, 0), (1, 1000003, 0, 0, 0),
])
def test_values_and_mask(kind, rows, cols, pad, first, offset):
    import torch
    code, dtype = TYPES[kind]
    ld = cols + pad
    for p, with_res in ((0.1, False), (0.5, True)):
        seed = 0x0123456789ABCDEF + rows
        x = matrix(torch, rows, cols, ld, dtype, 1, offset)
        r = matrix(torch, rows, cols, ld, dtype, 2, offset) if with_res else None
        yb = torch.full((rows, ld), 7.0, dtype=getattr(torch, dtype), device="cuda")
        cdl.cdl_dropout(x, ld, r, ld, yb, ld, code, rows, cols, p, seed, first)
        check(torch, yb[:, :cols], x, r, kept(first, rows, cols, seed, p), p)
        assert bool((yb[:, cols:] == 7.0).all())          # nothing between the rows is written


@pytest.mark.parametrize("kind", list(TYPES))
def test_probabilities_at_the_ends(kind):
    import torch
    code, dtype = TYPES[kind]
    x = matrix(torch, 9, 100, 100, dtype, 3)
    x[0, 0] = float("nan")
    x[1, 1] = float("inf")
    y = torch.empty_like(x)
    cdl.cdl_dropout(x, 100, None, 0, y, 100, code, 9, 100, 0.0, 5)
    assert torch.equal(torch.nan_to_num(y, nan=9.0), torch.nan_to_num(x, nan=9.0))
    cdl.cdl_dropout(x, 100, None, 0, y, 100, code, 9, 100, 1.0, 5)
    assert bool((y == 0).all())                            # a dropped NaN or infinity is 0
    big = float(np.float32(1.0 - 2.0 ** -24))              # the largest probability below 1: one word in 2^24 is kept
    cdl.cdl_dropout(x, 100, None, 0, y, 100, code, 9, 100, big, 5)
    assert int((y != 0).sum()) == int(kept(0, 9, 100, 5, big).sum())


def test_in_place_partition_and_backward():
    import torch
    rows, cols, p, seed = 50, 301, 0.25, 77
    x = matrix(torch, rows, cols, cols, "float32", 4).contiguous()
    y = torch.empty_like(x)
    cdl.cdl_dropout(x, cols, None, 0, y, cols, cdl.CDL_F32, rows, cols, p, seed, 10)
    z = x.clone()
    for r0, r1 in ((0, 13), (13, 14), (14, 50)):            # row ranges continue the counter space
        cdl.cdl_dropout(z[r0:], cols, None, 0, z[r0:], cols, cdl.CDL_F32, r1 - r0, cols, p, seed, 10 + r0 * cols)
    assert torch.equal(y, z)
    # backward: the same map on the gradient; the map is linear, so a difference quotient equals it up to rounding
    g = matrix(torch, rows, cols, cols, "float32", 5).contiguous()
    dx = torch.empty_like(g)
    cdl.cdl_dropout(g, cols, None, 0, dx, cols, cdl.CDL_F32, rows, cols, p, seed, 10)
    mask = torch.from_numpy(kept(10, rows, cols, seed, p)).cuda()
    assert bool(((dx != 0) <= mask).all())
    d = matrix(torch, rows, cols, cols, "float32", 6).contiguous()
    up = torch.empty_like(x)
    cdl.cdl_dropout(x + d, cols, None, 0, up, cols, cdl.CDL_F32, rows, cols, p, seed, 10)
    lhs = float((g.double() * (up.double() - y.double())).sum())
    rhs = float((dx.double() * d.double()).sum())
    size = float((g.abs() * (x.abs() + d.abs())).double().sum()) * 2
    assert abs(lhs - rhs) <= 4 * 2.0 ** -24 * size


def test_other_stream_and_empty():
    import torch
    x = matrix(torch, 64, 256, 256, "bfloat16", 8).contiguous()
    ref, y = torch.empty_like(x), torch.empty_like(x)
    cdl.cdl_dropout(x, 256, None, 0, ref, 256, cdl.CDL_BF16, 64, 256, 0.3, 9)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    cdl.cdl_dropout(x, 256, None, 0, y, 256, cdl.CDL_BF16, 64, 256, 0.3, 9, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(ref, y)
    assert cdl.cdl_dropout(None, 0, None, 0, None, 0, cdl.CDL_F32, 0, 5, 0.3, 9) == 0
    assert cdl.cdl_dropout(None, 0, None, 0, None, 0, cdl.CDL_F32, 5, 0, 0.3, 9) == 0


def test_counter_word_carries_into_the_next():
    """Blocks on both sides of a multiple of 2^32, at an even and at an odd place of a thread's two."""
    import torch
    for first in (4 * (2 ** 32 - 8), 4 * (2 ** 32 - 7), 4 * (5 * 2 ** 32 - 1), 4 * (2 ** 62 - 3)):
        x = matrix(torch, 1, 256, 256, "float32", 11)
        y = torch.empty_like(x)
        cdl.cdl_dropout(x, 256, None, 0, y, 256, cdl.CDL_F32, 1, 256, 0.5, 3, first)
        check(torch, y, x, None, kept(first, 1, 256, 3, 0.5), 0.5)


def test_more_elements_than_one_launch_takes():
    import torch
    n = (1 << 28) + 1003                                  # a single row: two launches of the vector form
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    cdl.cdl_dropout(x, n, None, 0, y, n, cdl.CDL_BF16, 1, n, 0.5, 21)
    at = (1 << 28) - 2000
    mask = torch.from_numpy(kept(at, 1, n - at, 21, 0.5)).cuda()[0]
    assert torch.equal(y[at:] != 0, mask)
    assert abs(float((y != 0).float().mean()) - 0.5) < 6 * 0.5 / n ** 0.5
