"""A softmax head learned on region descriptors: the rows that densenet_region_windows (or densenet_region_pool) returns,
normalised, against a vocabulary of classes or words.

    y = norm(descriptors) gamma;  loss = mean softmax cross entropy of y over w;  AdamW on gamma and w

Weights are kept in fp32 with a 16-bit copy for the products, which the optimiser writes as it steps: AdamW, or for w Muon.
``store`` gives descriptors in 8 bits with a scale, a quarter of their size.  ``step_8bit`` takes a step whose products read 8-bit
operands (blocks of 128 with a scale each), and ``answer`` gives each region's most probable words from such a product.

    python -m paper_1404_1869_amd.region_head [--words V] [--boxes N] [--steps K] [--muon] [--eight]

trains a head to tell the regions of a synthetic image apart, prints its loss and how many regions it answers right.
"""
from __future__ import annotations

import argparse
import math

from . import densenet as D


class RegionHead:
    """The head's parameters, gradients' buffers (times ``scale``) and optimiser states on one GPU."""

    def __init__(self, words: int, length: int = 9216, dtype: int = D.DN_BF16, state_bits: int = 8, eps: float = 1e-6, seed: int = 0,
                 device="cuda", muon: bool = False):
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
        # (Muon's update has singular values of about 1: a rate of 1 for each word's row to turn as fast as lr says)
        self.muon = D.MuonPlan([self.w], [self.dw], copies=copies, rates=[1.0]) if muon else None
        self.plans = (() if muon else (D.AdamWPlan([self.w], [self.dw], copies=copies, state_bits=state_bits),)) + \
            (D.AdamWPlan([self.gamma], [self.dgamma], state_bits=32),)

    def loss(self, descriptors, labels):
        """Loss of each row (0 where its label is outside the vocabulary)."""
        y, _, _ = D.densenet_rms_norm(descriptors, self.gamma, eps=self.eps, out_dtype=self.dtype)
        return D.densenet_softmax_loss(y, self.products, labels)[0]

    def step(self, descriptors, labels, lr: float = 2e-4, weight_decay: float = 0.01):
        """One training step on the mean loss of the rows that have a label.  Returns the rows' losses before it."""
        y, _, _ = D.densenet_rms_norm(descriptors, self.gamma, eps=self.eps, out_dtype=self.dtype)
        loss, lse = D.densenet_softmax_loss(y, self.products, labels)
        dy, _ = D.densenet_softmax_loss_backward(y, self.products, labels, lse, scale=self.scale, dw=self.dw)
        self._update(dy, descriptors, lr, weight_decay)
        return loss

    def _update(self, dy, descriptors, lr, weight_decay):
        """gamma's gradient, and the optimisers' steps."""
        D.densenet_rms_norm_backward(dy, descriptors, self.gamma, eps=self.eps, dgamma=self.dgamma)
        self.steps += 1
        for plan in self.plans:
            D.densenet_adamw(plan, lr=lr, step=self.steps, weight_decay=weight_decay, grad_scale=1 / self.scale, seed=self.steps)
        if self.muon:
            D.densenet_muon(self.muon, lr=lr, weight_decay=weight_decay, grad_scale=1 / self.scale)

    def words_8bit(self, turned: bool = False):
        """w's codes and scales in squares of 128 (and turned, for dy), for answers until w changes."""
        return D.densenet_quantize_blocks(self.products, rows=D.DN_SCALE_BLOCK, turned=turned)

    def step_8bit(self, descriptors, labels, lr: float = 2e-4, weight_decay: float = 0.01):
        """As ``step``, all products reading 8-bit operands: logits of the rows' codes and w's, dy of the logits' gradient's codes
        and w's turned ones, dw of both turned ones.  Returns the rows' losses before it."""
        import torch
        y, _, _ = D.densenet_rms_norm(descriptors, self.gamma, eps=self.eps, out_dtype=self.dtype)
        codes, scale, _, _ = D.densenet_quantize_blocks(y)
        _, _, turned, turned_scale = D.densenet_quantize_blocks(y, rows=D.DN_SCALE_BLOCK, codes=False, turned=True)
        w, w_scale, wt, wt_scale = self.words_8bit(turned=True)
        logits = D.densenet_block_product(codes, scale, w, w_scale, out_dtype=self.dtype)
        logp, _, lse, _, _ = D.densenet_token_scores(logits, labels)
        has = (labels >= 0) & (labels < self.w.shape[0])
        dlogp = torch.where(has, -self.scale / has.sum().clamp(min=1), 0.0).float()
        g = D.densenet_token_scores_backward(logits, labels, lse, dlogp=dlogp, out=logits)
        g, g_scale, gt, gt_scale = D.densenet_quantize_blocks(g, turned=True)
        dy = D.densenet_block_product(g, g_scale, wt, wt_scale, out_dtype=self.dtype)
        D.densenet_block_product(gt, gt_scale, turned, turned_scale, out_dtype=self.dtype, out=self.dw)
        self._update(dy, descriptors, lr, weight_decay)
        return -logp

    def answer(self, descriptors, top: int = 5, words=None):
        """Each row's `top` most probable words, their log probabilities, and the entropy of its distribution, from products in 8
        bits of normalised rows that are 8-bit codes from the start.  words: of ``words_8bit``, which a caller keeps between answers
        (by default made anew)."""
        codes, _, scale = D.densenet_rms_norm(descriptors, self.gamma, eps=self.eps, out_dtype=D.DN_F8, block=D.DN_SCALE_BLOCK)
        w, w_scale = (words or self.words_8bit())[:2]
        logits = D.densenet_block_product(codes, scale, w, w_scale, out_dtype=self.dtype)
        _, entropy, _, ids, logp = D.densenet_token_scores(logits, top=top)
        return ids, logp, entropy

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
    ap.add_argument("--muon", action="store_true", help="step w by Muon instead of AdamW")
    ap.add_argument("--eight", action="store_true", help="products in 8 bits")
    args = ap.parse_args(argv)
    if min(args.words, args.boxes, args.steps) < 1:
        ap.error("--words, --boxes and --steps must be at least 1")
    desc = image_descriptors(args.boxes)
    labels = torch.arange(args.boxes, device="cuda") % args.words
    head = RegionHead(args.words, desc.shape[1], muon=args.muon)
    for k in range(args.steps):
        loss = (head.step_8bit if args.eight else head.step)(desc, labels)
        print(f"step {k + 1}: loss {float(loss.mean()):.4f}", flush=True)
    ids, _, entropy = head.answer(desc)
    print(f"{int((ids[:, 0] == labels).sum())} of {args.boxes} regions answered right, mean entropy {float(entropy.mean()):.3f}")
    codes, scale = head.store(desc)
    print(f"{args.boxes} descriptors: {desc.numel() * 4 >> 20} MiB in fp32, {(codes.numel() + 4 * scale.numel()) >> 20} MiB stored in 8 bits")
    return float(loss.mean())


if __name__ == "__main__":
    main()
