"""A softmax head learned on region descriptors: the rows that densenet_region_windows (or densenet_region_pool) returns,
normalised, against a vocabulary of classes or words.

    y = norm(descriptors) gamma;  loss = mean softmax cross entropy of y over w;  AdamW on gamma and w

Weights are kept in fp32 with a 16-bit copy for the products, which the optimiser writes as it steps.  ``store`` gives
descriptors in 8 bits with a scale, a quarter of their size.

    python -m paper_1404_1869_amd.region_head [--words V] [--boxes N] [--steps K]

trains a head to tell the regions of a synthetic image apart and prints its loss.
"""
from __future__ import annotations

import argparse
import math

from . import densenet as D


class RegionHead:
    """The head's parameters, gradients' buffers (times ``scale``) and optimiser states on one GPU."""

    def __init__(self, words: int, length: int = 9216, dtype: int = D.DN_BF16, state_bits: int = 8, eps: float = 1e-6, seed: int = 0,
                 device="cuda"):
        import torch
        g = torch.Generator(device=device).manual_seed(seed)
        self.dtype, self.eps, self.steps = dtype, eps, 0
        self.gamma = torch.ones(length, device=device)
        self.w = torch.randn(words, length, generator=g, device=device) * (0.1 / length ** 0.5)
        low = D._tdtype(dtype)
        self.products = self.w if dtype == D.DN_F32 else self.w.to(low)  # what the products read
        # fp16's gradients of a mean over many rows are next to nothing: they are taken times a power of two, and the optimiser
        # divides by it.  A row of y is at most sqrt(length) |gamma|, and so dw at most half of fp16's range times |gamma|.
        self.scale = 2.0 ** math.floor(math.log2(32768 / length ** 0.5)) if dtype == D.DN_F16 else 1.0
        self.dgamma, self.dw = torch.zeros_like(self.gamma), torch.zeros(words, length, dtype=low, device=device)
        copies = None if dtype == D.DN_F32 else [self.products]
        self.plans = (D.AdamWPlan([self.w], [self.dw], copies=copies, state_bits=state_bits),
                      D.AdamWPlan([self.gamma], [self.dgamma], state_bits=32))

    def loss(self, descriptors, labels):
        """Loss of each row (0 where its label is outside the vocabulary)."""
        y, _, _ = D.densenet_rms_norm(descriptors, self.gamma, eps=self.eps, out_dtype=self.dtype)
        return D.densenet_softmax_loss(y, self.products, labels)[0]

    def step(self, descriptors, labels, lr: float = 2e-4, weight_decay: float = 0.01):
        """One training step on the mean loss of the rows that have a label.  Returns the rows' losses before it."""
        y, _, _ = D.densenet_rms_norm(descriptors, self.gamma, eps=self.eps, out_dtype=self.dtype)
        loss, lse = D.densenet_softmax_loss(y, self.products, labels)
        dy, _ = D.densenet_softmax_loss_backward(y, self.products, labels, lse, scale=self.scale, dw=self.dw)
        D.densenet_rms_norm_backward(dy, descriptors, self.gamma, eps=self.eps, dgamma=self.dgamma)
        self.steps += 1
        for plan in self.plans:
            D.densenet_adamw(plan, lr=lr, step=self.steps, weight_decay=weight_decay, grad_scale=1 / self.scale, seed=self.steps)
        return loss

    def store(self, descriptors):
        """Normalised descriptors as 8-bit codes and a scale for each row: value = code * scale."""
        codes, _, scale = D.densenet_rms_norm(descriptors, self.gamma, eps=self.eps, out_dtype=D.DN_F8)
        return codes, scale


def image_descriptors(n_boxes: int, seed: int = 11):
    """Descriptors of n_boxes regions of a synthetic 480 x 640 image, from its 8-scale pyramid (fp16)."""
    import torch

    from . import configs, synth
    w = configs.VGA_8SCALE
    p = D.params_for(w)
    packed = D.densenet_pack_weights([(torch.from_numpy(a).cuda(), torch.from_numpy(b).cuda()) for a, b in synth.weights(7)], D.DN_F16)
    pyra = D.convnet_featpyramid(torch.from_numpy(synth.image(seed, w.H, w.W)).cuda(), p, packed, D.DN_F16)
    boxes = torch.from_numpy(synth.boxes(seed, n_boxes, w.H, w.W)).cuda()
    return D.densenet_region_windows(pyra.conv.conv5, list(pyra.conv.c5d), D.DN_F16, pyra.plan, w.pad, len(pyra.plan.planes), boxes)[0]


def main(argv=None):
    import torch
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--words", type=int, default=1000)
    ap.add_argument("--boxes", type=int, default=2000)
    ap.add_argument("--steps", type=int, default=20)
    args = ap.parse_args(argv)
    if min(args.words, args.boxes, args.steps) < 1:
        ap.error("--words, --boxes and --steps must be at least 1")
    desc = image_descriptors(args.boxes)
    labels = torch.arange(args.boxes, device="cuda") % args.words
    head = RegionHead(args.words, desc.shape[1])
    for k in range(args.steps):
        loss = head.step(desc, labels)
        print(f"step {k + 1}: loss {float(loss.mean()):.4f}", flush=True)
    codes, scale = head.store(desc)
    print(f"{args.boxes} descriptors: {desc.numel() * 4 >> 20} MiB in fp32, {(codes.numel() + 4 * scale.numel()) >> 20} MiB stored in 8 bits")
    return float(loss.mean())


if __name__ == "__main__":
    main()
