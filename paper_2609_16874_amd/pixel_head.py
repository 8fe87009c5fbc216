"""A pixel head that ends in the decoder: residual blocks, if any, group norm with
an activation, then the projections to the embedding map and to its foreground
plane, forward and backward through the HIP operators of ``head`` and ``rows8``.

``python -m paper_2609_16874_amd.pixel_head`` trains one on a synthetic frame
(the target is Eq1's encoding of each pixel's centroid) and decodes what it
then says, printing the share of labelled pixels before and after, and after with
the trained head in 8-bit integers.  ``--blocks N`` puts N residual blocks before
the norm, ``--checkpoint8`` keeps activations for the gradient in 8 bits.
"""
from __future__ import annotations

import argparse

import torch

from . import head, native, rows8, synth
from .pixel_block import PixelBlock, PixelBlock8


class PixelHead:
    """Handles and parameters of a head for frames of ``H`` x ``W`` pixels with
    ``channels`` features, writing D embedding channels and a foreground plane
    in the layout that ``native.Decoder`` reads (dtype "f16" or "f32"), after
    ``blocks`` residual blocks of twice the features; ``checkpoint8``: what
    ``backward`` needs of the blocks and of the projections' input is kept in 8 bits."""

    def __init__(self, H: int, W: int, channels: int, groups: int, D: int, dtype: str = "f16",
                 activation: str = "silu", seed: int = 0, blocks: int = 0, checkpoint8: bool = False):
        self.H, self.W, self.D, self.dtype, self.activation, self.checkpoint8 = H, W, D, dtype, activation, checkpoint8
        self.blocks = [PixelBlock(H * W, channels, 2 * channels, dtype, activation, checkpoint8, seed + 1 + i)
                       for i in range(blocks)]
        self.norm = head.GroupNorm(1, H * W, channels, groups, dtype, activation)
        self.to_emb = head.Linear(H * W, channels, D, dtype)
        self.to_fg = head.Linear(H * W, channels, 1, dtype)
        t = native.torch_dtype(dtype)
        g = torch.Generator().manual_seed(seed)

        def weight(n):
            return (torch.randn((n, channels), generator=g) * channels ** -0.5).to(t).cuda()

        self.params = {"gamma": torch.ones(channels, device="cuda"), "beta": torch.zeros(channels, device="cuda"),
                       "w_emb": weight(D), "b_emb": torch.zeros(D, device="cuda"),
                       "w_fg": weight(1), "b_fg": torch.zeros(1, device="cuda")}
        for i, b in enumerate(self.blocks):
            self.params.update({f"block{i}.{k}": v for k, v in b.params.items()})
        self._kept = None

    def forward(self, features):
        """(emb [H][W][D], fg [H][W]) of features [H][W][channels]; keeps what
        ``backward`` needs."""
        p = self.params
        features = _through(self.blocks, features)
        hidden, stats = self.norm.run(features[None], p["gamma"], p["beta"])
        rows = hidden.view(self.H * self.W, -1)
        emb = self.to_emb.run(rows, p["w_emb"], p["b_emb"])
        fg = self.to_fg.run(rows, p["w_fg"], p["b_fg"])
        self._kept = (features, stats, rows8.packed(rows) if self.checkpoint8 else rows)
        return emb.view(self.H, self.W, self.D), fg.view(self.H, self.W)

    def backward(self, d_emb, d_fg):
        """Gradients by the parameters' names, and "features", of the last
        ``forward`` from those of its outputs."""
        p, (features, stats, rows) = self.params, self._kept
        d_emb, d_fg = d_emb.reshape(-1, self.D), d_fg.reshape(-1, 1)
        if self.checkpoint8:
            d_rows, dw_emb, db_emb = self.to_emb.run_backward8(*rows, p["w_emb"], d_emb)
            d_rows_fg, dw_fg, db_fg = self.to_fg.run_backward8(*rows, p["w_fg"], d_fg)
        else:
            d_rows, dw_emb, db_emb = self.to_emb.run_backward(rows, p["w_emb"], d_emb)
            d_rows_fg, dw_fg, db_fg = self.to_fg.run_backward(rows, p["w_fg"], d_fg)
        d_rows += d_rows_fg
        d_x, d_gamma, d_beta = self.norm.run_backward(features[None], d_rows.view(1, self.H * self.W, -1),
                                                      p["gamma"], p["beta"], stats)
        grads = {"gamma": d_gamma, "beta": d_beta, "w_emb": dw_emb, "b_emb": db_emb, "w_fg": dw_fg, "b_fg": db_fg}
        d = d_x[0]
        for i in reversed(range(len(self.blocks))):     # (a block's output and its stream are added: one gradient)
            d = d.reshape(self.H * self.W, -1)
            of_block = self.blocks[i].backward(d, d)
            d = of_block.pop("x")
            grads.update({f"block{i}.{k}": v for k, v in of_block.items()})
        return {**grads, "features": d.reshape(features.shape)}

    def close(self):
        for op in (self.norm, self.to_emb, self.to_fg, *self.blocks):
            op.close()


class PixelHead8:
    """A trained ``PixelHead`` for serving: the products of its blocks and its
    projections in 8-bit integers."""

    def __init__(self, trained: PixelHead):
        h, p = trained, trained.params
        self.H, self.W, self.D = h.H, h.W, h.D
        channels = h.norm.channels
        self.blocks = [PixelBlock8(b) for b in h.blocks]
        self.norm = head.GroupNorm(1, h.H * h.W, channels, h.norm.groups, h.dtype, h.activation)
        self.gamma, self.beta = p["gamma"].clone(), p["beta"].clone()
        self.to_emb = rows8.Linear8(h.H * h.W, channels, h.D, h.dtype)
        self.to_fg = rows8.Linear8(h.H * h.W, channels, 1, h.dtype)
        self.w_emb, self.w_fg = rows8.packed(p["w_emb"]), rows8.packed(p["w_fg"])
        self.b_emb, self.b_fg = p["b_emb"].clone(), p["b_fg"].clone()

    def forward(self, features):
        """(emb, fg), as the trained head's."""
        features = _through(self.blocks, features)
        hidden, _ = self.norm.run(features[None], self.gamma, self.beta)
        q, scale = rows8.packed(hidden.view(self.H * self.W, -1))
        emb = self.to_emb.run(q, scale, *self.w_emb, self.b_emb)
        fg = self.to_fg.run(q, scale, *self.w_fg, self.b_fg)
        return emb.view(self.H, self.W, self.D), fg.view(self.H, self.W)

    def close(self):
        for op in (self.norm, self.to_emb, self.to_fg, *self.blocks):
            op.close()


def _through(blocks, features):
    """Features [H][W][channels] after the blocks."""
    x, residual = features.reshape(-1, features.shape[-1]), None
    for b in blocks:
        x, residual = b.forward(x, residual)
    return features if residual is None else (x + residual).view(features.shape)


def features_of(frame, channels: int, noise: float = 0.05, seed: int = 1):
    """Stand-in backbone features of a synthetic frame: a fixed random mixture
    of its clean encoding and foreground, and noise."""
    spec = frame.spec
    fx, fy = spec.freqs()
    clean = torch.zeros((spec.H, spec.W, spec.D + 1))
    inside = torch.from_numpy(frame.inst > 0)
    table = synth.encode_positions(frame.centroids[:, 0], frame.centroids[:, 1], fx, fy)
    clean[..., :spec.D][inside] = torch.from_numpy(table).float()[torch.from_numpy(frame.inst).long()[inside] - 1]
    clean[..., spec.D] = inside.float()
    g = torch.Generator().manual_seed(seed)
    mix = torch.randn((spec.D + 1, channels), generator=g) * (spec.D + 1) ** -0.5
    x = clean @ mix + noise * torch.randn((spec.H, spec.W, channels), generator=g)
    return x.to(native.torch_dtype(spec.dtype)).cuda(), clean.cuda(), inside.cuda()


def train(head_, features, target, inside, steps: int, rate: float = 0.02):
    """Steps of Adam on the mean squared error of the embedding (foreground
    pixels) and of the foreground plane; the losses."""
    moments = {k: (torch.zeros_like(v, dtype=torch.float32), torch.zeros_like(v, dtype=torch.float32))
               for k, v in head_.params.items()}
    master = {k: v.float() for k, v in head_.params.items()}
    count = inside.sum()
    losses = []
    for step in range(1, steps + 1):
        emb, fg = head_.forward(features)
        off_emb = (emb.float() - target[..., :-1]) * inside[..., None]
        off_fg = fg.float() - target[..., -1]
        losses.append(off_emb.square().sum() / (count * head_.D) + off_fg.square().mean())
        # scaled so that the 16-bit gradients do not underflow; Adam divides the scale out
        grads = head_.backward((off_emb * (1024.0 / head_.D)).to(emb.dtype), (off_fg * 256.0).to(fg.dtype))
        for k, m in master.items():
            a, b = moments[k]
            g = grads[k].float()
            a.lerp_(g, 0.1)
            b.lerp_(g * g, 0.01)
            m -= rate * (a / (1 - 0.9 ** step)) / ((b / (1 - 0.99 ** step)).sqrt() + 1e-8)
            head_.params[k].copy_(m)
    return [float(v) for v in losses]


def agreement(labels, inst) -> float:
    """Share of the instances' pixels whose label is the one that most pixels
    of their instance have, and that has most of its pixels there."""
    import numpy as np
    K, N = int(labels.max()), int(inst.max())
    both = np.bincount(inst.ravel().astype(np.int64) * (K + 1) + labels.ravel(), minlength=(N + 1) * (K + 1))
    both = both.reshape(N + 1, K + 1)
    best = both[1:, 1:].argmax(1) + 1 if K else np.zeros(N, dtype=np.int64)
    right = sum(int(both[i + 1, k]) for i, k in enumerate(best) if k and both[1:, k].argmax() == i)
    return right / max(1, int((inst > 0).sum()))


def main(config: int = 1, channels: int = 64, steps: int = 150, blocks: int = 0, checkpoint8: bool = False):
    frame = synth.make_frame(config)
    spec = frame.spec
    fx, fy = spec.freqs()
    features, target, inside = features_of(frame, channels)
    pixel_head = PixelHead(spec.H, spec.W, channels, 8, spec.D, spec.dtype, blocks=blocks, checkpoint8=checkpoint8)
    dec = native.Decoder(spec.H, spec.W, spec.n_freq, spec.dtype, fx, fy, spec.bins, spec.bins)
    peak = 2.5 * spec.H * spec.W / 256.0 ** 2

    def decoded(with_head):
        out = dec.run(*with_head.forward(features), spec.fg_threshold, peak, score=False)
        return out["K"], agreement(out["labels"], frame.inst)

    before = decoded(pixel_head)
    losses = train(pixel_head, features, target, inside, steps)
    after = decoded(pixel_head)
    served = PixelHead8(pixel_head)
    in_8_bits = decoded(served)
    served.close()
    print(f"{spec.name}: loss {losses[0]:.3f} -> {losses[-1]:.4f} in {steps} steps; of {len(frame.centroids)} "
          f"instances {before[0]} -> {after[0]} centroids, {before[1]:.1%} -> {after[1]:.1%} of the pixels right "
          f"({in_8_bits[1]:.1%} in 8 bits)")
    dec.close()
    pixel_head.close()
    return losses, before, after


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description="Trains a pixel head on a synthetic frame and decodes its output.")
    parser.add_argument("--blocks", type=int, default=0)
    parser.add_argument("--checkpoint8", action="store_true")
    arguments = parser.parse_args()
    main(blocks=arguments.blocks, checkpoint8=arguments.checkpoint8)
