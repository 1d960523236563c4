"""The feed-forward half of a transformer's block in 8-bit floating point, run and trained on one GPU:

    s = x + residual, norm of s, as codes      patdnn_rms_norm
    silu(gate) * up, as codes                  patdnn_fp8_gated
    back to the stream                         patdnn_fp8_linear

so a pass is three launches (and a small one for few rows); its result and s are the next block's x and residual.  ``Block.gradients`` is the backward pass as a training
program calls it: every product on codes, quantised along the axis that it sums over, gradients of weights in fp32.  Weights are random.
``python -m paper_2001_00138_amd.examples.feed_forward`` prints how long a token, a prompt and a training step take.
"""

from __future__ import annotations

import time

from paper_2001_00138_amd import binding as B


class Block:
    def __init__(self, width: int, hidden: int, seed: int = 0, eps: float = 1e-6):
        import torch
        g = torch.Generator(device="cuda").manual_seed(seed)
        random = lambda *shape: torch.randn(shape, generator=g, device="cuda")      # noqa: E731
        self.width, self.hidden, self.eps = width, hidden, eps
        self.gamma = 1 + 0.1 * random(width)
        self.both = (random(2 * hidden, width) * width ** -0.5).bfloat16()          # gate's rows, then up's
        self.down = (random(width, hidden) * hidden ** -0.5).bfloat16()
        self.quantise()

    def quantise(self):
        """Codes of the weights for a pass, and of their transposes (the same squares' scales) for the gradients; after every change of the weights."""
        squares = dict(blocks="squares")
        self.gate, self.gate_scales = B.patdnn_fp8_quantize(self.both[:self.hidden], **squares)
        self.up, self.up_scales = B.patdnn_fp8_quantize(self.both[self.hidden:], **squares)
        self.down8 = B.patdnn_fp8_quantize(self.down, **squares)
        self.both_t = B.patdnn_fp8_quantize(self.both, transposed=True, **squares)
        self.down_t = B.patdnn_fp8_quantize(self.down, transposed=True, **squares)

    def __call__(self, x, residual=None, keep=None):
        """x, residual [rows, width] bfloat16 -> (the block's result, the stream that it is to be added to).  ``keep``: a dict that gets what the backward pass needs."""
        codes, scales, stream, rstd = B.patdnn_rms_norm(x, self.gamma, residual=residual, eps=self.eps, fp8=True)
        h, h_scales = B.patdnn_fp8_gated(codes, scales, self.gate, self.gate_scales, self.up, self.up_scales, fp8=True)
        out = B.patdnn_fp8_linear(h, h_scales, *self.down8, dtype=x.dtype)
        if keep is not None:
            keep.update(codes=codes, scales=scales, stream=stream, rstd=rstd, h=h, h_scales=h_scales)
        return out, stream

    def gradients(self, kept, dout, dstream=None):
        """-> dict of the gradients of x (and residual: the same), gamma, both [2 * hidden, width] and down, from those of a pass's two results."""
        import torch
        rows = dout.shape[0]
        dout8 = B.patdnn_fp8_quantize(dout)
        dh = B.patdnn_fp8_linear(*dout8, *self.down_t, dtype=dout.dtype)
        d_both = B.patdnn_fp8_gated_backward(dh, kept["codes"], kept["scales"], self.gate, self.gate_scales, self.up, self.up_scales)
        d_normed = B.patdnn_fp8_linear(*B.patdnn_fp8_quantize(d_both), *self.both_t, dtype=dout.dtype)
        # sums over rows: both sides quantised along them
        along_rows = lambda t: B.patdnn_fp8_quantize(t, transposed=True)            # noqa: E731
        normed = B.patdnn_fp8_dequantize(kept["codes"], kept["scales"], self.width, dtype=torch.bfloat16)
        h = B.patdnn_fp8_dequantize(kept["h"], kept["h_scales"], self.hidden, dtype=torch.bfloat16)
        g_both = B.patdnn_fp8_linear(*along_rows(d_both), *along_rows(normed)) if rows else torch.zeros_like(self.both, dtype=torch.float32)
        g_down = B.patdnn_fp8_linear(*along_rows(dout), *along_rows(h)) if rows else torch.zeros_like(self.down, dtype=torch.float32)
        dx, dgamma = B.patdnn_rms_norm_backward(d_normed, kept["stream"], kept["rstd"], self.gamma, dsum=dstream)
        return {"x": dx, "gamma": dgamma, "both": g_both, "down": g_down}


def main() -> None:
    import torch
    block = Block(4096, 12288)

    def timed(f, times=20):
        for _ in range(3):
            f()
        torch.cuda.synchronize()
        began = time.perf_counter()
        for _ in range(times):
            f()
        torch.cuda.synchronize()
        return (time.perf_counter() - began) / times * 1e6

    for rows in (1, 64, 8192):
        x, residual = (torch.randn(rows, block.width, device="cuda").bfloat16() for _ in range(2))
        print(f"{rows} row(s): {timed(lambda: block(x, residual)):.0f} us a pass")
    kept = {}
    out, stream = block(x, residual, kept)
    print(f"gradients of {rows} rows: {timed(lambda: block.gradients(kept, out, stream)):.0f} us")


if __name__ == "__main__":
    main()
