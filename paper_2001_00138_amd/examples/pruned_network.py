"""A small residual-free network of pattern-pruned convolutions, run end to end on one GPU:

    3x3 convolution, pruned (fp32, NCHW, bias)       patdnn_conv2d
    to channels last, fp16                           patdnn_channels_last
    group norm + SiLU                                patdnn_group_norm
    pointwise layer, MXFP4 weights, bias + ReLU      patdnn_mxfp4_linear, rows are pixels
    back to NCHW, fp32                               patdnn_channels_first

as often as ``WIDTHS`` says, a last pruned convolution with ReLU and 2x2 pooling, and a classifier on the flattened planes (MXFP4 again).
Weights are random.  ``python -m paper_2001_00138_amd.examples.pruned_network`` prints what it stores and how long a pass takes;
``Network(...).normalisation_gradients`` is the backward pass through one normalisation, as a program that tunes
gamma and beta of a pruned network calls it.
"""

from __future__ import annotations

import time

import numpy as np

from paper_2001_00138_amd import binding as B
from paper_2001_00138_amd import workloads as wl

WIDTHS = (16, 32, 64)            # channels of the input and behind each block
GROUPS, CLASSES = 8, 100


class Network:
    def __init__(self, side: int = 28, seed: int = 0):
        import torch
        rng = np.random.default_rng(seed)
        library = wl.pattern_library(wl.PATTERN_SEED)

        def pruned(c_in, c_out):
            w = rng.standard_normal((c_out, c_in, 3, 3)).astype(np.float32) * np.float32(np.sqrt(2 / (9 * c_in)))
            ids, w = B.patdnn_project_patterns(w, library)                    # the pruning stage's projections
            mask = B.patdnn_project_connectivity(w, c_out * c_in // 2)
            return B.Layer(w, ids, mask, library), torch.from_numpy(rng.standard_normal(c_out).astype(np.float32) * 0.1).cuda()

        def linear(features, out):
            w = torch.from_numpy(rng.standard_normal((out, features)).astype(np.float32) * np.float32(np.sqrt(2 / features))).cuda()
            bias = torch.from_numpy(rng.standard_normal(out).astype(np.float32) * np.float32(0.1)).cuda()
            return (*B.patdnn_mxfp4_quantize(w), bias)

        self.blocks = []
        for c_in, c_out in zip(WIDTHS[:-1], WIDTHS[1:]):
            gamma = torch.from_numpy(1 + 0.2 * rng.standard_normal(c_in).astype(np.float32)).cuda()
            beta = torch.from_numpy(0.2 * rng.standard_normal(c_in).astype(np.float32)).cuda()
            self.blocks.append((pruned(c_in, c_in), gamma, beta, linear(c_in, c_out)))
        self.last = pruned(WIDTHS[-1], WIDTHS[-1])
        self.classifier = linear(WIDTHS[-1] * (side // 2) ** 2, CLASSES)
        self.side = side

    def __call__(self, x, keep=None):
        """x [n, WIDTHS[0], side, side] fp32 -> logits [n, CLASSES] fp32.  ``keep``: a list that gets (name, tensor) of every step."""
        import torch
        keep = [] if keep is None else keep
        for (layer, bias), gamma, beta, (w, scales, b) in self.blocks:
            x = layer.conv2d(x, bias)
            keep.append(("conv", x))
            h = B.patdnn_channels_last(x, dtype=torch.float16)
            keep.append(("last", h))
            h, mean, rstd = B.patdnn_group_norm(h, GROUPS, gamma, beta, act="silu")
            keep.extend([("norm", h), ("mean", mean), ("rstd", rstd)])
            n, rows, cols, c = h.shape
            h = B.patdnn_mxfp4_linear(h.view(-1, c), w, scales, b, act="relu").view(n, rows, cols, -1)
            keep.append(("pointwise", h))
            x = B.patdnn_channels_first(h, dtype=torch.float32)
            keep.append(("first", x))
        layer, bias = self.last
        x = layer.conv2d_pool(x, bias)
        keep.append(("pool", x))
        w, scales, b = self.classifier
        x = B.patdnn_mxfp4_linear(x.view(x.shape[0], -1), w, scales, b)
        keep.append(("logits", x))
        return x

    def normalisation_gradients(self, block: int, h, mean, rstd, dy):
        """(dx, dgamma, dbeta) of block's normalisation, for its fp16 input h and the gradient dy of its output."""
        _, gamma, beta, _ = self.blocks[block]
        return B.patdnn_group_norm_backward(dy, h, mean, rstd, GROUPS, gamma, beta, act="silu")

    def close(self):
        for (layer, _), _, _, _ in self.blocks:
            layer.close()
        self.last[0].close()


def main() -> None:
    import torch
    net = Network()
    w, scales, _ = net.classifier
    print(f"classifier: {CLASSES} x {w.shape[1] * 2} weights in {w.numel() + scales.numel()} bytes")
    for n in (1, 64):
        x = torch.randn(n, WIDTHS[0], net.side, net.side, device="cuda")
        for _ in range(3):
            net(x)
        torch.cuda.synchronize()
        began = time.perf_counter()
        for _ in range(20):
            net(x)
        torch.cuda.synchronize()
        print(f"{n} image(s): {(time.perf_counter() - began) / 20 * 1e6:.0f} us a pass")
    net.close()


if __name__ == "__main__":
    main()
