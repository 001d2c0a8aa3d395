"""How the linear layers' sums are taken: the same result with a checkpoint and without, and errors that do not grow with the reduced extent, in every
form of the kernels."""
import math

import pytest

import paper_2501_09849_b200 as cdl
from linear_plan import forward_form, tile_plan

pytestmark = pytest.mark.gpu
TYPES = {"f32": (cdl.CDL_F32, "float32"), "bf16": (cdl.CDL_BF16, "bfloat16"), "f16": (cdl.CDL_F16, "float16")}


def up(n, m):
    return -(-n // m) * m


def operand(torch, rows, cols, kind, std, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    m = torch.full((rows, up(cols, 8)), float("nan"), dtype=getattr(torch, TYPES[kind][1]), device="cuda")
    m[:, :cols] = (torch.randn(rows, cols, generator=g, device="cuda") * std).to(m.dtype)
    return m


class Forward:
    def __init__(self, torch, kind, M, N, K):
        self.torch, self.code, self.M, self.N, self.K = torch, TYPES[kind][0], M, N, K
        self.a, self.w = operand(torch, M, K, kind, 1.0, 1), operand(torch, N, K, kind, 1 / math.sqrt(K), 2)
        self.b, self.nb = torch.randn(N, generator=torch.Generator().manual_seed(3)).cuda(), cdl.cdl_linear_workspace_bytes(M, N, K)
        self.ws = torch.empty(self.nb, dtype=torch.uint8, device="cuda")

    def run(self, out, act=cdl.CDL_ACT_NONE, bias=True, keep=False):
        t, M, N = self.torch, self.M, self.N
        o = t.empty(M, N, dtype=getattr(t, TYPES[out][1]), device="cuda")
        codes, scales = (t.zeros(M, up(N, 16), dtype=t.uint8, device="cuda"), t.empty(-(-N // 128), M, device="cuda")) if keep else (None, None)
        cdl.cdl_linear_fwd(self.a, self.a.stride(0), self.w, self.w.stride(0), self.code, self.b if bias else None, act, None, 0, M, N, self.K, o, N, TYPES[out][0],
                           codes, up(N, 16) if keep else 0, scales, ws=self.ws, ws_bytes=self.nb)
        cdl.cdl_workspace_status(self.ws)
        return (o, codes, scales) if keep else o

    def exact(self):
        return self.a[:, :self.K].double() @ self.w[:, :self.K].double().t()


# one size or more for each form, all with more reduced entries than are summed in one go
SIZES = [(8, 1000, 3000, "rows"), (3, 30000, 2280, "rows"), (100, 300, 5000, "cluster"), (300, 300, 20000, "singles with runs"), (1100, 2000, 1100, "singles"),
         (2000, 2304, 1500, "pairs"), (2300, 2304, 5000, "pairs with runs"), (4100, 3000, 1090, "pairs")]


@pytest.mark.parametrize("kind,out", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("M,N,K,form", SIZES)
def test_a_result_does_not_depend_on_its_checkpoint(kind, out, M, N, K, form):
    import torch
    assert forward_form(M, N, K) == form
    f = Forward(torch, kind, M, N, K)
    for act in (cdl.CDL_ACT_NONE, cdl.CDL_ACT_GELU):
        plain, (kept, _, _) = f.run(out, act), f.run(out, act, keep=True)
        assert torch.equal(plain, kept)


@pytest.mark.parametrize("M,N,K,form", [s for s in SIZES if s[3] != "rows"])
def test_errors_do_not_grow_with_the_reduced_extent(M, N, K, form):
    """For random signs an instruction's cut shortens a sum by 2^-24.5 of itself on average, so n instructions by n / 2 * 2^-24.5: 32 of them for
    binary32 results 6.8e-7 of the norm, 64 for the scales of a 16-bit result's checkpoint 1.35e-6.  What is added rounded is far below."""
    import torch
    f = Forward(torch, "bf16", M, N, K)
    ref = f.exact()
    assert float((f.run("f32", bias=False).double() - ref).norm() / ref.norm()) <= 7e-7
    gb = -(-N // 128)
    largest = torch.nn.functional.pad(ref.abs(), (0, gb * 128 - N)).view(M, gb, 128).amax(2).t() / 448
    for out, bound in (("f32", 7e-7), ("bf16", 1.4e-6)):
        scales = f.run(out, bias=False, keep=True)[2].double()
        assert float((scales - largest).norm() / largest.norm()) <= bound, out


@pytest.mark.parametrize("M,N,K,form", [(8192, 512, 256, "cluster"), (50000, 130, 72, "singles with runs"), (6000, 2304, 2304, "pairs with runs")])
def test_weight_gradients_over_many_rows(M, N, K, form):
    """The same bound for binary32 weight gradients; 16-bit ones are those of sums that are 1.4e-6 off at most, so that all but a few in a thousand are
    the correctly rounded ones: an entry of binary16 is rounded the other way where it lies as near to a border, which are 2^-10 to 2^-11 of it apart."""
    import torch
    assert tile_plan(N, K, M).form == form
    dy, a = operand(torch, M, N, "f16", 1.0, 1), operand(torch, M, K, "f16", 1.0, 2)
    nb = cdl.cdl_linear_workspace_bytes(M, N, K)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    ref = dy[:, :N].double().t() @ a[:, :K].double()
    for out in ("f32", "f16"):
        dw = torch.empty(N, K, dtype=getattr(torch, TYPES[out][1]), device="cuda")
        cdl.cdl_linear_bwd_weight(dy, dy.stride(0), a, a.stride(0), cdl.CDL_F16, M, N, K, False, dw, K, TYPES[out][0], ws=ws, ws_bytes=nb)
        if out == "f32":
            assert float((dw.double() - ref).norm() / ref.norm()) <= 7e-7
        else:
            # errors of standard deviation 1.4e-6 of the norm's entry, against a border every 2^-11 of the entry or more: 1.4e-6 * 2^11 = 0.3 %, thrice that
            # for entries below the norm's
            assert float((dw != ref.half()).double().mean()) <= 0.01


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("M,N,K", [(8, 1000, 3000), (3, 4655, 40000), (8, 4655, 60000), (5, 30000, 2280)])
def test_few_rows(kind, M, N, K):
    """The same bound where one to eight rows have a form of their own, whose warps take up to 7500 reduced entries each here."""
    import torch
    assert forward_form(M, N, K) == "rows"
    f = Forward(torch, kind, M, N, K)
    ref = f.exact()
    assert float((f.run("f32", bias=False).double() - ref).norm() / ref.norm()) <= 7e-7
    gb = -(-N // 128)
    largest = torch.nn.functional.pad(ref.abs(), (0, gb * 128 - N)).view(M, gb, 128).amax(2).t() / 448
    scales = f.run(kind, bias=False, keep=True)[2].double()
    assert float((scales - largest).norm() / largest.norm()) <= 1.4e-6
