"""Residual blocks over a map's pixels, through the HIP operators: RMS norm with
the residual stream's addition, a product with an activation, a product back.

A block takes the last one's output and the stream before it, (x, residual), and
returns its own output and the stream, (y, sum): the next norm adds the two, so
the stream is read and written once a block.  ``PixelBlock`` trains, with its
activations kept for the gradient as they are or in 8 bits (``checkpoint8``: half
the memory or a quarter from a block's forward to its backward; while the forward
runs its own activations are there as they are, too); ``PixelBlock8`` serves a
trained one in integers.
"""
from __future__ import annotations

import torch

from . import head, native, rows8
from .head import _unrecorded


class PixelBlock:
    """Handles and parameters of a block over up to ``rows`` pixels of
    ``channels`` features, ``hidden`` of them between its products."""

    def __init__(self, rows: int, channels: int, hidden: int, dtype: str = "f16", activation: str = "silu",
                 checkpoint8: bool = False, seed: int = 0):
        self.rows, self.channels, self.hidden, self.dtype, self.activation = rows, channels, hidden, dtype, activation
        self.checkpoint8 = checkpoint8
        self.norm = rows8.RmsNorm(rows, channels, dtype)
        self.up = head.Linear(rows, channels, hidden, dtype, activation)
        self.down = head.Linear(rows, hidden, channels, dtype)
        t = native.torch_dtype(dtype)
        g = torch.Generator().manual_seed(seed)

        def weight(n, k):
            return (torch.randn((n, k), generator=g) * k ** -0.5).to(t).cuda()

        self.params = {"gamma": torch.ones(channels, device="cuda"), "w_up": weight(hidden, channels),
                       "b_up": torch.zeros(hidden, device="cuda"), "w_down": weight(channels, hidden),
                       "b_down": torch.zeros(channels, device="cuda")}
        self._kept = None

    def forward(self, x, residual=None):
        """(y, sum) of x [rows][channels] and the stream before it (none: x
        begins it); keeps what ``backward`` needs.  Not recorded by autograd:
        tensors that require a gradient are refused while it records."""
        p = self.params
        _unrecorded("PixelBlock.forward", x, residual, p["gamma"])
        total = x if residual is None else torch.empty_like(x)
        u = torch.empty_like(x)
        rstd = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
        q, scale = (torch.empty(x.shape, dtype=torch.int8, device=x.device), torch.empty_like(rstd)) \
            if self.checkpoint8 else (None, None)
        st = self.norm.forward(x, p["gamma"], residual, None if residual is None else total, u, q, scale, rstd)
        if st != native.CPE_OK:
            raise native.CpeError(st, "cpe_rms_forward")
        h, z = self.up.run(u, p["w_up"], p["b_up"], keep=True)
        y = self.down.run(h, p["w_down"], p["b_down"])
        if self.checkpoint8:
            self._kept = (rows8.packed(total), (q, scale), rows8.packed(z), rows8.packed(h), rstd)
        else:
            self._kept = (total, u, z, h, rstd)
        return y, total

    def backward(self, d_y, d_sum):
        """Gradients by the parameters' names, and "x" (which is the residual's
        as well), of the last ``forward`` from those of its outputs."""
        p, (total, u, z, h, rstd) = self.params, self._kept
        if self.checkpoint8:
            d_h, dw_down, db_down = self.down.run_backward8(*h, p["w_down"], d_y)
            d_u, dw_up, db_up = self.up.run_backward8(*u, p["w_up"], d_h, *z)
            d_x, d_gamma = self.norm.run_backward(total[0], d_u, p["gamma"], rstd, d_sum, total[1])
        else:
            d_h, dw_down, db_down = self.down.run_backward(h, p["w_down"], d_y)
            d_u, dw_up, db_up = self.up.run_backward(u, p["w_up"], d_h, z)
            d_x, d_gamma = self.norm.run_backward(total, d_u, p["gamma"], rstd, d_sum)
        return {"gamma": d_gamma, "w_up": dw_up, "b_up": db_up, "w_down": dw_down, "b_down": db_down, "x": d_x}

    def kept_bytes(self) -> int:
        """What the last ``forward`` keeps for the gradient."""
        tensors = [t for k in self._kept for t in (k if isinstance(k, tuple) else (k,))]
        return sum(t.numel() * t.element_size() for t in tensors)

    def close(self):
        for op in (self.norm, self.up, self.down):
            op.close()


class PixelBlock8:
    """A trained block for serving: its products in 8-bit integers, the weights
    with a scale for each output feature, packed here."""

    def __init__(self, block: PixelBlock):
        b = block
        self.norm = rows8.RmsNorm(b.rows, b.channels, b.dtype)
        self.up = rows8.Linear8(b.rows, b.channels, b.hidden, b.dtype, b.activation)
        self.down = rows8.Linear8(b.rows, b.hidden, b.channels, b.dtype)
        self.gamma, self.b_up, self.b_down = (b.params[k].clone() for k in ("gamma", "b_up", "b_down"))
        self.w_up, self.w_down = rows8.packed(b.params["w_up"]), rows8.packed(b.params["w_down"])

    def forward(self, x, residual=None):
        """(y, sum), as the trained block's."""
        if residual is None:
            total, ((q, scale), _) = x, self.norm.run(x, self.gamma, packed=True)
        else:
            total, (q, scale), _ = self.norm.run(x, self.gamma, residual, packed=True)
        h = self.up.run(q, scale, *self.w_up, self.b_up)
        return self.down.run(*rows8.packed(h), *self.w_down, self.b_down), total

    def close(self):
        for op in (self.norm, self.up, self.down):
            op.close()
