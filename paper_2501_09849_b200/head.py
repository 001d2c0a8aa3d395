"""One training step of a language model's output head on the library's calls: an 8-bit linear layer, dropout with the
residual connection, and the cross entropy over a vocabulary, forward and backward.

Like layer.CdlLayerStep this module only owns device buffers and issues the calls in order on one stream (recordable into a
CUDA graph); every number but the bias' gradient is produced by the kernels behind the ABI.

Step (x: T x D hidden states, labels: T words, W1: D x D layer weights in binary32, W2: V x D output weights):
   1  W1 -> e4m3 codes, a scale per 128 x 128 block, both orientations               cdl_fp8_quantize
   2  x  -> codes, a scale per 128 entries, along rows and along tokens                cdl_fp8_quantize
   3  Y = X W1^T + b                                                                   cdl_fp8_matmul
   4  H = dropout(Y) + x                                                               cdl_dropout
   5  loss, lse of H W2^T against the labels                                            cdl_vocab_loss_fwd
   6  dH, dW2 for dloss (1 / count for a mean)                                          cdl_vocab_loss_bwd
   7  dY = dropout(dH): the same map, drawn again                                       cdl_dropout
   8  dY -> codes along rows and along tokens                                           cdl_fp8_quantize
   9  dX = dY W1 (W1's transposed codes), then + dH of the residual connection          cdl_fp8_matmul, cdl_dropout with p = 0
  10  dW1 = dY^T X                                                                      cdl_fp8_matmul
  11  db1 = column sums of dY, with a bias                                                torch.sum
The optimizer is outside.

``python -m paper_2501_09849_b200.head`` trains such a head on a synthetic task for a few steps and prints the loss.
"""
from __future__ import annotations

from . import api as cdl


def _up(n, m=16):
    return -(-n // m) * m


class HeadStep:
    def __init__(self, torch, T, D, V, p=0.1, seed=0, bias=False, device="cuda"):
        if D % 8:
            raise ValueError("the width of the hidden states is a multiple of 8")
        self.torch, self.T, self.D, self.V, self.p, self.seed = torch, T, D, V, float(p), int(seed)
        t, f32, bf16, f8 = torch, torch.float32, torch.bfloat16, torch.float8_e4m3fn

        def empty(shape, dtype):
            return t.empty(shape, dtype=dtype, device=device)
        kb, tb = -(-D // 128), -(-T // 128)
        # inputs of a step
        self.x, self.labels = empty((T, D), bf16), empty((T,), t.int64)
        self.w1, self.w2 = empty((D, D), f32), empty((V, D), bf16)
        self.b1 = t.zeros(D, dtype=f32, device=device) if bias else None
        self.dloss = t.full((T,), 1.0 / max(T, 1), dtype=f32, device=device)
        # 8-bit operands: codes with their scales, and the transposed ones
        self.w1c, self.w1s = empty((D, _up(D)), f8), empty((kb, kb), f32)
        self.w1ct, self.w1st = empty((D, _up(D)), f8), empty((kb, kb), f32)
        self.xc, self.xs = empty((T, _up(D)), f8), empty((kb, T), f32)
        self.xct, self.xst = empty((D, _up(T)), f8), empty((tb, D), f32)
        self.gc, self.gs = empty((T, _up(D)), f8), empty((kb, T), f32)
        self.gct, self.gst = empty((D, _up(T)), f8), empty((tb, D), f32)
        # results
        self.y, self.h = empty((T, D), bf16), empty((T, D), bf16)
        self.loss, self.lse = empty((T,), f32), empty((T,), f32)
        self.dh, self.dy, self.dx = empty((T, D), bf16), empty((T, D), bf16), empty((T, D), bf16)
        self.dw1, self.dw2 = empty((D, D), f32), empty((V, D), bf16)
        self.db1 = empty((D,), f32) if bias else None
        self.ws_bytes = max(cdl.cdl_fp8_matmul_workspace_bytes(T, D, D), cdl.cdl_fp8_matmul_workspace_bytes(D, D, T),
                            cdl.cdl_vocab_loss_workspace_bytes(T, V, D, True))
        self.ws = empty((self.ws_bytes,), t.uint8)

    def run(self, first_index=0):
        """Enqueues one step.  first_index: the first element of this step's dropout in the counter space of `seed`; T * D elements
        are used."""
        T, D, V = self.T, self.D, self.V
        rows, blocks, bf16, f32 = cdl.CDL_FP8_ROWS, cdl.CDL_FP8_BLOCKS, cdl.CDL_BF16, cdl.CDL_F32
        pd, pt, ws = _up(D), _up(T), dict(ws=self.ws, ws_bytes=self.ws_bytes)
        cdl.cdl_fp8_quantize(self.w1, D, f32, D, D, blocks, self.w1c, pd, self.w1s, self.w1ct, pd, self.w1st)
        cdl.cdl_fp8_quantize(self.x, D, bf16, T, D, rows, self.xc, pd, self.xs, self.xct, pt, self.xst)
        cdl.cdl_fp8_matmul(self.xc, pd, self.xs, self.w1c, pd, self.w1s, blocks, T, D, D, self.y, D, bf16, self.b1, **ws)
        cdl.cdl_dropout(self.y, D, self.x, D, self.h, D, bf16, T, D, self.p, self.seed, first_index)
        cdl.cdl_vocab_loss_fwd(self.h, D, self.w2, D, bf16, self.labels, T, V, D, self.loss, self.lse, **ws)
        cdl.cdl_vocab_loss_bwd(self.h, D, self.w2, D, bf16, self.labels, self.lse, self.dloss, T, V, D, self.dh, D, self.dw2, D, **ws)
        cdl.cdl_dropout(self.dh, D, None, 0, self.dy, D, bf16, T, D, self.p, self.seed, first_index)
        cdl.cdl_fp8_quantize(self.dy, D, bf16, T, D, rows, self.gc, pd, self.gs, self.gct, pt, self.gst)
        cdl.cdl_fp8_matmul(self.gc, pd, self.gs, self.w1ct, pd, self.w1st, blocks, T, D, D, self.dx, D, bf16, **ws)
        cdl.cdl_dropout(self.dx, D, self.dh, D, self.dx, D, bf16, T, D, 0.0, self.seed)
        cdl.cdl_fp8_matmul(self.gct, pt, self.gst, self.xct, pt, self.xst, rows, D, D, T, self.dw1, D, f32, **ws)
        if self.db1 is not None:
            self.torch.sum(self.dy, 0, dtype=self.torch.float32, out=self.db1)

    def capture(self):
        """Records one step into a CUDA graph and returns it.  A replay draws the same dropout again: this is for a step whose
        inputs change and whose mask may stay, such as a measurement, or p = 0."""
        t = self.torch
        graph, side = t.cuda.CUDAGraph(), t.cuda.Stream()
        side.wait_stream(t.cuda.current_stream())
        with t.cuda.stream(side):
            self.run()                  # the library's one-time set-up per device must not fall into the capture
            side.synchronize()
            with t.cuda.graph(graph, stream=side):
                self.run()
        t.cuda.current_stream().wait_stream(side)
        return graph


def main(steps=40, T=512, D=256, V=4000, rate=0.02):
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    step = HeadStep(torch, T, D, V, p=0.1, seed=7)
    step.x.copy_(torch.randn(T, D, generator=g, device="cuda"))
    step.labels.copy_(torch.randint(0, V, (T,), generator=g, device="cuda"))
    step.w1.copy_(torch.randn(D, D, generator=g, device="cuda") / D ** 0.5)
    w2 = torch.randn(V, D, generator=g, device="cuda") / D ** 0.5
    for k in range(steps):
        step.w2.copy_(w2)
        step.run(first_index=k * T * D)
        step.w1.sub_(rate * step.dw1)
        w2.sub_(rate * T * step.dw2.float())
        if k % 5 == 0 or k == steps - 1:
            print(f"step {k:3d}  loss {float(step.loss.mean()):.4f}")
    cdl.cdl_workspace_status(step.ws)


if __name__ == "__main__":
    main()
