"""Refusals of the language-model operators: every bad argument is answered by its status before anything is enqueued, on a
machine without a device as well (an enqueue attempt there would come back as a launch error)."""
import pytest

import paper_2501_09849_b200 as cdl
from paper_2501_09849_b200 import build as cdl_build

ARG, ALIGN, RANGE, WS = -1, -2, -3, -4
P = 0x10000          # a pointer that is never followed


@pytest.fixture(scope="module", autouse=True)
def lib():
    cdl_build.build()
    return cdl.load_library()


def test_dropout_refusals():
    def f(x=P, ldx=64, r=None, ldr=0, y=P, ldy=64, type=cdl.CDL_F32, rows=3, cols=64, p=0.1):
        return cdl.cdl_dropout(x, ldx, r, ldr, y, ldy, type, rows, cols, p, 1, check=False)
    assert f(x=None) == ARG and f(y=None) == ARG and f(type=3) == ARG and f(type=-1) == ARG
    assert f(rows=-1) == ARG and f(cols=-1) == ARG and f(ldx=63) == ARG and f(ldy=63) == ARG and f(r=P, ldr=63) == ARG
    assert f(rows=2 ** 40, cols=2 ** 40, ldx=2 ** 40, ldy=2 ** 40) == ARG
    assert f(p=-0.1) == RANGE and f(p=1.5) == RANGE and f(p=float("nan")) == RANGE
    assert f(x=P + 2) == ALIGN and f(y=P + 1) == ALIGN and f(r=P + 2, ldr=64) == ALIGN and f(x=P + 1, type=cdl.CDL_BF16) == ALIGN
    assert f(rows=0, x=None, y=None) == 0 and f(cols=0, x=None, y=None) == 0
    with pytest.raises(cdl.CdlError):
        cdl.cdl_dropout(P, 8, None, 0, P, 8, cdl.CDL_F32, 1, 8, 2.0, 1)


def test_fp8_quantize_refusals():
    def f(x=P, ldx=100, type=cdl.CDL_BF16, rows=30, cols=100, mode=cdl.CDL_FP8_ROWS, codes=P, ldc=112, s=P, ct=None, ldt=0, st=None):
        return cdl.cdl_fp8_quantize(x, ldx, type, rows, cols, mode, codes, ldc, s, ct, ldt, st, check=False)
    assert f(x=None) == ARG and f(codes=None) == ARG and f(s=None) == ARG and f(type=5) == ARG and f(mode=2) == ARG
    assert f(rows=-1) == ARG and f(cols=-1) == ARG and f(ldx=99) == ARG and f(ldc=96) == ARG
    assert f(ct=P) == ARG and f(st=P) == ARG and f(ct=P, st=P, ldt=16) == ARG
    assert f(x=P + 1) == ALIGN and f(x=P + 2, type=cdl.CDL_F32) == ALIGN and f(codes=P + 8) == ALIGN and f(ldc=104) == ALIGN and f(s=P + 2) == ALIGN
    assert f(ct=P + 8, st=P, ldt=32) == ALIGN and f(ct=P, st=P, ldt=40) == ALIGN and f(ct=P, st=P + 1, ldt=32) == ALIGN
    assert f(rows=2 ** 31 - 1, cols=2 ** 31 - 1, ldx=2 ** 31, ldc=2 ** 31) == ARG          # more tiles than a launch has blocks
    assert f(cols=2 ** 30 + 1, ldx=2 ** 31, ldc=2 ** 31) == ARG
    assert f(rows=0) == 0 and f(cols=0) == 0


def test_fp8_matmul_refusals():
    n = cdl.cdl_fp8_matmul_workspace_bytes(30, 100, 200)
    assert n >= 256 and cdl.cdl_fp8_matmul_workspace_bytes(-1, 1, 1) == 0

    def f(A=P, lda=208, sa=P, B=P, ldb=208, sb=P, mode=cdl.CDL_FP8_BLOCKS, M=30, N=100, K=200, out=P, ldo=100, type=cdl.CDL_BF16, bias=None, ws=P, nb=n):
        return cdl.cdl_fp8_matmul(A, lda, sa, B, ldb, sb, mode, M, N, K, out, ldo, type, bias, ws, nb, check=False)
    assert f(A=None) == ARG and f(B=None) == ARG and f(sa=None) == ARG and f(sb=None) == ARG and f(out=None) == ARG
    assert f(mode=7) == ARG and f(type=3) == ARG and f(M=-1) == ARG and f(N=-1) == ARG and f(K=-1) == ARG
    assert f(lda=192) == ARG and f(ldb=192) == ARG and f(ldo=99) == ARG
    assert f(A=P + 8) == ALIGN and f(B=P + 8) == ALIGN and f(lda=204) == ALIGN and f(ldb=204) == ALIGN and f(out=P + 1) == ALIGN
    assert f(sa=P + 2) == ALIGN and f(sb=P + 2) == ALIGN and f(bias=P + 2) == ALIGN and f(out=P + 2, type=cdl.CDL_F32) == ALIGN
    assert f(ws=None) == WS and f(ws=P + 16) == WS and f(nb=n - 1) == WS
    assert f(K=2 ** 30 + 1, lda=2 ** 31, ldb=2 ** 31) == ARG and cdl.cdl_fp8_matmul_workspace_bytes(1, 2 ** 30 + 1, 1) == 0
    assert f(M=0) == 0 and f(N=0) == 0


def test_vocab_loss_refusals():
    n0, n1 = cdl.cdl_vocab_loss_workspace_bytes(30, 1000, 72, 0), cdl.cdl_vocab_loss_workspace_bytes(30, 1000, 72, 1)
    assert 256 <= n0 <= n1
    assert cdl.cdl_vocab_loss_workspace_bytes(-1, 10, 8, 0) == 0 and cdl.cdl_vocab_loss_workspace_bytes(1, 0, 8, 0) == 0 and cdl.cdl_vocab_loss_workspace_bytes(1, 10, 0, 0) == 0

    def f(H=P, ldh=72, W=P, ldw=72, type=cdl.CDL_BF16, y=P, T=30, V=1000, D=72, loss=P, lse=P, ws=P, nb=n0):
        return cdl.cdl_vocab_loss_fwd(H, ldh, W, ldw, type, y, T, V, D, loss, lse, ws, nb, check=False)

    def b(H=P, ldh=72, W=P, ldw=72, type=cdl.CDL_BF16, y=P, lse=P, g=P, T=30, V=1000, D=72, dH=P, lddh=72, dW=P, lddw=72, ws=P, nb=n1):
        return cdl.cdl_vocab_loss_bwd(H, ldh, W, ldw, type, y, lse, g, T, V, D, dH, lddh, dW, lddw, ws, nb, check=False)
    for call in (f, b):
        assert call(H=None) == ARG and call(W=None) == ARG and call(y=None) == ARG and call(lse=None) == ARG
        assert call(type=cdl.CDL_F32) == ARG and call(type=9) == ARG
        assert call(V=2 ** 30 + 1) == ARG
        assert call(T=-1) == ARG and call(V=0) == ARG and call(D=0) == ARG and call(ldh=64) == ARG and call(ldw=64) == ARG
        assert call(H=P + 8) == ALIGN and call(W=P + 8) == ALIGN and call(ldh=76) == ALIGN and call(ldw=76) == ALIGN and call(y=P + 4) == ALIGN
        assert call(lse=P + 2) == ALIGN
        assert call(ws=None) == WS and call(ws=P + 64) == WS
    assert f(loss=None) == ARG and f(loss=P + 1) == ALIGN and f(nb=n0 - 1) == WS
    assert b(g=None) == ARG and b(lddh=64) == ARG and b(lddw=64) == ARG and b(nb=n1 - 1) == WS
    assert b(dH=P + 8) == ALIGN and b(dW=P + 8) == ALIGN and b(lddh=76) == ALIGN and b(lddw=76) == ALIGN and b(g=P + 1) == ALIGN
    assert f(T=0, H=None, y=None) == 0
