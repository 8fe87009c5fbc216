"""ctypes binding of the head operators (``include/cpe_head.h``): group norm
with an activation over channels-last maps and the matrix product with bias,
activation and residual, each with its gradient.

Argument marshalling only, like ``native``: device buffers are torch tensors,
their pointers, strides and torch's current HIP stream are passed through.
Calls return the C ABI's status; ``native.CpeError`` is raised by the
constructors and by the ``run`` conveniences.  A tensor whose shape, dtype or
device the C ABI could not see is refused here with ``ValueError``.

``stream`` stands for ``with torch.cuda.stream(stream)`` around the call: what
``run`` and ``run_backward`` allocate belongs to it.  Inputs that another
stream writes, and outputs that another stream reads, are ordered by the caller.
"""
from __future__ import annotations

import contextlib
import ctypes
from typing import Optional

import torch

from .native import CPE_OK, CpeError, library, torch_dtype

DTYPES = {"f32": 0, "f16": 1, "bf16": 2}
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}


def _stream(stream, device: int) -> int:
    """The HIP stream's handle (the current one's without the stream object,
    whose construction takes as long as the launch)."""
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream


def _allocating(stream):
    """New tensors are taken from the pool of the stream that writes them: a
    block of the current stream's pool may have work on it that is still to run."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _unrecorded(what: str, *tensors):
    """``run`` is no node of autograd's graph: a gradient asked for through it
    would be lost without a word."""
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError(f"{what} is not recorded by autograd: call it under torch.no_grad() or on detached "
                                 "tensors, and run_backward for the gradient")


def _int32(v, what: str) -> int:
    """A size as the C ABI's int32, which ctypes would cut off without a word."""
    v = int(v)
    _need(-(1 << 31) <= v < 1 << 31, f"{what}: {v} is no 32-bit size")
    return v


def _vector(t, n: int, name: str, device: int, dtype=torch.float32):
    """The pointer of a contiguous device vector, or None."""
    if t is None:
        return None
    if not (t.get_device() == device and t.dtype is dtype and t.numel() == n and t.is_contiguous()):
        raise ValueError(f"{name}: a contiguous tensor of {n} {dtype} on the handle's device is needed")
    return t.data_ptr()


class GroupNorm:
    """Handle of one group norm (channels, groups, dtype, activation) for
    calls of up to ``max_samples`` samples of ``max_pixels`` pixels.  Maps are
    [samples][pixels][C] tensors (or [samples][H][W][C] ones whose rows follow
    one another) with contiguous channels; other strides are free."""
    _device = None      # the handle's; a host tensor's get_device() is -1

    def __init__(self, max_samples: int, max_pixels: int, channels: int, groups: int, dtype: str,
                 activation: str = "none", eps: float = 1e-5):
        self.channels, self.groups, self.dtype = _int32(channels, "channels"), _int32(groups, "groups"), dtype
        self.eps, self._torch_dtype, self._lib = float(eps), torch_dtype(dtype), library()
        h = ctypes.c_void_p()
        st = self._lib.cpe_norm_create(ctypes.byref(h), _int32(max_samples, "max_samples"),
                                       _int32(max_pixels, "max_pixels"), self.channels, self.groups,
                                       DTYPES[dtype], ACTIVATIONS[activation], self.eps)
        if st != CPE_OK:
            raise CpeError(st, "cpe_norm_create")
        self._h, self._device = h, torch.cuda.current_device()

    def _map(self, t, name: str, size=None):
        """(pointer, pixel stride, sample stride, (samples, pixels)) of a map."""
        shape, strides = t.shape, t.stride()
        if len(shape) == 3:
            samples, pixels, channels = shape
            ld = strides[1]
        else:
            _need(len(shape) == 4, f"{name}: three or four dimensions, channels last")
            samples, height, width, channels = shape
            pixels = height * width
            # (the stride of a dimension of one says nothing: a column's pixels are its image rows)
            _need(height <= 1 or width <= 1 or strides[1] == width * strides[2],
                  f"{name}: image rows must follow one another")
            ld = strides[2] if width > 1 else strides[1]
        if not (t.get_device() == self._device and t.dtype is self._torch_dtype and channels == self.channels
                and (channels == 1 or strides[-1] == 1) and (size is None or size == (samples, pixels))):
            raise ValueError(f"{name}: wrong shape, dtype, device or channel stride")
        if pixels <= 1 and ld < channels:      # the stride of a single pixel says nothing
            ld = channels
        if size is None and (samples >> 31 or pixels >> 31):
            raise ValueError(f"{name}: {samples} x {pixels} are no 32-bit sizes")
        return t.data_ptr(), ld, strides[0], (samples, pixels)

    def forward(self, x, gamma, beta, y, stats=None, valid=None, stream=None) -> int:
        """cpe_norm_forward: ``stats`` receives float32 [samples][G][2] for the
        gradient; ``valid`` holds int32 pixel counts, one per sample."""
        px, x_ld, x_sample, size = self._map(x, "x")
        py, y_ld, y_sample, _ = self._map(y, "y", size)
        dev = self._device
        return self._lib.cpe_norm_forward(
            self._h, _stream(stream, dev), size[0], size[1], px, x_ld, x_sample,
            _vector(gamma, self.channels, "gamma", dev), _vector(beta, self.channels, "beta", dev),
            _vector(valid, size[0], "valid", dev, torch.int32), py, y_ld, y_sample,
            _vector(stats, 2 * size[0] * self.groups, "stats", dev))

    def backward(self, x, dy, gamma, beta, stats, dx=None, dgamma=None, dbeta=None, valid=None, stream=None) -> int:
        """cpe_norm_backward: writes those of dx, dgamma and dbeta that are given."""
        px, x_ld, x_sample, size = self._map(x, "x")
        pd, dy_ld, dy_sample, _ = self._map(dy, "dy", size)
        po, dx_ld, dx_sample, _ = (None, 0, 0, None) if dx is None else self._map(dx, "dx", size)
        dev = self._device
        return self._lib.cpe_norm_backward(
            self._h, _stream(stream, dev), size[0], size[1], px, x_ld, x_sample, pd, dy_ld, dy_sample,
            _vector(gamma, self.channels, "gamma", dev), _vector(beta, self.channels, "beta", dev),
            _vector(valid, size[0], "valid", dev, torch.int32),
            _vector(stats, 2 * size[0] * self.groups, "stats", dev), po, dx_ld, dx_sample,
            _vector(dgamma, self.channels, "dgamma", dev), _vector(dbeta, self.channels, "dbeta", dev))

    def run(self, x, gamma, beta, valid=None, stream=None):
        """forward into new tensors: (y, stats).  Not recorded by autograd:
        tensors that require a gradient are refused while it records."""
        _unrecorded("GroupNorm.run", x, gamma, beta)
        with _allocating(stream):
            y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
            stats = torch.empty((x.shape[0], self.groups, 2), dtype=torch.float32, device=x.device)
            if x.numel() == 0:      # the call has nothing to do: what it says of samples without pixels
                stats[..., 0] = 0.0
                stats[..., 1] = self.eps ** -0.5
        st = self.forward(x, gamma, beta, y, stats, valid, stream)
        if st != CPE_OK:
            raise CpeError(st, "cpe_norm_forward")
        return y, stats

    def run_backward(self, x, dy, gamma, beta, stats, valid=None, stream=None):
        """backward into new tensors: (dx, dgamma, dbeta)."""
        with _allocating(stream):
            dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
            dgamma, dbeta = (torch.empty(self.channels, dtype=torch.float32, device=x.device) for _ in range(2))
        st = self.backward(x, dy, gamma, beta, stats, dx, dgamma, dbeta, valid, stream)
        if st != CPE_OK:
            raise CpeError(st, "cpe_norm_backward")
        return dx, dgamma, dbeta

    def workspace_bytes(self) -> int:
        return int(self._lib.cpe_norm_workspace_bytes(self._h))

    def close(self):
        if getattr(self, "_h", None):
            self._lib.cpe_norm_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Linear:
    """Handle of one matrix product (features, dtype, activation) for calls of
    up to ``max_rows`` rows.  Matrices are [rows][features] tensors with
    contiguous features and any row stride; the weight is [out][in]."""
    _device = None      # the handle's; a host tensor's get_device() is -1

    def __init__(self, max_rows: int, in_features: int, out_features: int, dtype: str, activation: str = "none"):
        self.in_features, self.out_features = _int32(in_features, "in_features"), _int32(out_features, "out_features")
        self.dtype = dtype
        self._torch_dtype, self._lib = torch_dtype(dtype), library()
        h = ctypes.c_void_p()
        st = self._lib.cpe_linear_create(ctypes.byref(h), _int32(max_rows, "max_rows"), self.in_features,
                                         self.out_features, DTYPES[dtype], ACTIVATIONS[activation])
        if st != CPE_OK:
            raise CpeError(st, "cpe_linear_create")
        self._h, self._device = h, torch.cuda.current_device()

    def _matrix(self, t, rows: Optional[int], width: int, name: str):
        """(pointer, row stride) of a matrix, (None, 0) for None."""
        if t is None:
            return None, 0
        shape, strides = t.shape, t.stride()
        if not (len(shape) == 2 and t.get_device() == self._device and t.dtype is self._torch_dtype
                and shape[1] == width and (rows is None or shape[0] == rows) and (width == 1 or strides[1] == 1)):
            raise ValueError(f"{name}: wrong shape, dtype, device or feature stride")
        ld = strides[0]
        return t.data_ptr(), width if shape[0] <= 1 and ld < width else ld

    def forward(self, x, weight, bias, y, residual=None, preact=None, stream=None) -> int:
        """cpe_linear_forward: ``preact`` receives the value before the
        activation, which the gradient needs."""
        rows, n = x.shape[0], self.out_features
        if rows >> 31:
            raise ValueError(f"x: {rows} is no 32-bit number of rows")
        px, x_ld = self._matrix(x, None, self.in_features, "x")
        pw, w_ld = self._matrix(weight, n, self.in_features, "weight")
        py, y_ld = self._matrix(y, rows, n, "y")
        pr, r_ld = self._matrix(residual, rows, n, "residual")
        pz, z_ld = self._matrix(preact, rows, n, "preact")
        return self._lib.cpe_linear_forward(self._h, _stream(stream, self._device), rows, px, x_ld, pw, w_ld,
                                            _vector(bias, n, "bias", self._device), pr, r_ld, py, y_ld, pz, z_ld)

    def backward(self, x, weight, dy, preact=None, dx=None, dweight=None, dbias=None, stream=None) -> int:
        """cpe_linear_backward: writes those of dx, dweight and dbias that are given."""
        rows, k, n = x.shape[0], self.in_features, self.out_features
        if rows >> 31:
            raise ValueError(f"x: {rows} is no 32-bit number of rows")
        px, x_ld = self._matrix(x, None, k, "x")
        pw, w_ld = self._matrix(weight, n, k, "weight")
        pd, d_ld = self._matrix(dy, rows, n, "dy")
        pz, z_ld = self._matrix(preact, rows, n, "preact")
        po, o_ld = self._matrix(dx, rows, k, "dx")
        pg, g_ld = self._matrix(dweight, n, k, "dweight")
        return self._lib.cpe_linear_backward(self._h, _stream(stream, self._device), rows, px, x_ld, pw, w_ld, pd, d_ld,
                                             pz, z_ld, po, o_ld, pg, g_ld,
                                             _vector(dbias, n, "dbias", self._device))

    def run(self, x, weight, bias=None, residual=None, keep=False, stream=None):
        """forward into new tensors: y, or (y, preact) where ``keep``.  Not
        recorded by autograd: tensors that require a gradient are refused while
        it records."""
        _unrecorded("Linear.run", x, weight, bias, residual)
        with _allocating(stream):
            y = torch.empty((x.shape[0], self.out_features), dtype=x.dtype, device=x.device)
            preact = torch.empty_like(y) if keep else None
        st = self.forward(x, weight, bias, y, residual, preact, stream)
        if st != CPE_OK:
            raise CpeError(st, "cpe_linear_forward")
        return (y, preact) if keep else y

    def run_backward(self, x, weight, dy, preact=None, stream=None):
        """backward into new tensors: (dx, dweight, dbias)."""
        with _allocating(stream):
            dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
            dweight = torch.empty(weight.shape, dtype=x.dtype, device=x.device)
            dbias = torch.empty(self.out_features, dtype=torch.float32, device=x.device)
        st = self.backward(x, weight, dy, preact, dx, dweight, dbias, stream)
        if st != CPE_OK:
            raise CpeError(st, "cpe_linear_backward")
        return dx, dweight, dbias

    def workspace_bytes(self) -> int:
        return int(self._lib.cpe_linear_workspace_bytes(self._h))

    def close(self):
        if getattr(self, "_h", None):
            self._lib.cpe_linear_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
