"""ctypes binding of the operators on rows held in 8 bits
(``include/cpe_rows8.h``): rows packed and unpacked, RMS norm with the
residual's addition that writes them, and the integer matrix product that reads
them.  ``head.Linear.backward8`` and ``RmsNorm.backward`` take checkpoints in
them.

Rows in 8 bits are an int8 [rows][width] tensor with contiguous elements and any
row stride, and a contiguous float32 [rows] tensor of scales: row r stands for
``q[r] * scale[r]``.  Argument marshalling only, with ``head``'s conventions for
streams, status codes and refusals.
"""
from __future__ import annotations

import ctypes

import torch

from .head import ACTIVATIONS, DTYPES, _allocating, _int32, _matrix, _stream, _unrecorded, _vector
from .native import CPE_OK, CpeError, library, torch_dtype

_CODES = {torch.float32: DTYPES["f32"], torch.float16: DTYPES["f16"], torch.bfloat16: DTYPES["bf16"]}


def _packed(q, scale, rows, width, name: str, device: int):
    """(pointer, row stride, pointer of the scales) of rows in 8 bits."""
    p, ld = _matrix(q, rows, width, name, device, torch.int8)
    return p, ld, _vector(scale, q.shape[0], "the scales", device)


def _current_device() -> int:
    """(torch.cuda.current_device without its check that the device is set up,
    which a tensor on it says)"""
    return torch._C._cuda_getDevice()


def _free_matrix(t, name: str):
    """(pointer, row stride, rows, width, device) of a matrix that no handle
    goes with, as the C ABI's sizes; its device has to be the current one."""
    shape, strides, device = t.shape, t.stride(), t.get_device()
    if len(shape) != 2 or shape[0] >> 31 or shape[1] >> 31 or (shape[1] != 1 and strides[1] != 1):
        raise ValueError(f"{name}: a matrix of 32-bit sizes and contiguous rows is needed")
    if device < 0 or device != _current_device():
        raise ValueError(f"{name}: a tensor on the current device is needed")
    rows, width = shape
    ld = strides[0]
    return t.data_ptr(), width if rows <= 1 and ld < width else ld, rows, width, device


def pack(x, q, scale, stream=None) -> int:
    """cpe_rows8_pack: writes the rows of ``x`` in 8 bits."""
    px, x_ld, rows, width, dev = _free_matrix(x, "x")
    code = _CODES.get(x.dtype)
    if code is None:
        raise ValueError("x: float32, float16 or bfloat16 is needed")
    pq, q_ld = _matrix(q, rows, width, "q", dev, torch.int8)
    return library().cpe_rows8_pack(_stream(stream, dev), rows, width, code, px, x_ld, pq, q_ld,
                                    _vector(scale, rows, "scale", dev))


def unpack(q, scale, x, stream=None) -> int:
    """cpe_rows8_unpack: writes the values that rows in 8 bits stand for, in
    the type of ``x``."""
    pq, q_ld, rows, width, dev = _free_matrix(q, "q")
    dtype = x.dtype
    code = _CODES.get(dtype)
    if code is None or q.dtype is not torch.int8:
        raise ValueError("q: int8, and x: float32, float16 or bfloat16 are needed")
    px, x_ld = _matrix(x, rows, width, "x", dev, dtype)
    return library().cpe_rows8_unpack(_stream(stream, dev), rows, width, pq, q_ld, _vector(scale, rows, "scale", dev),
                                      code, px, x_ld)


def packed(x, stream=None):
    """pack into new tensors: (q, scale)."""
    _unrecorded("rows8.packed", x)
    with _allocating(stream):
        q = torch.empty(x.shape, dtype=torch.int8, device=x.device)
        scale = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
    st = pack(x, q, scale, stream)
    if st != CPE_OK:
        raise CpeError(st, "cpe_rows8_pack")
    return q, scale


def unpacked(q, scale, dtype: str, stream=None):
    """unpack into a new tensor of the dtype ("f32", "f16", "bf16")."""
    with _allocating(stream):
        x = torch.empty(q.shape, dtype=torch_dtype(dtype), device=q.device)
    st = unpack(q, scale, x, stream)
    if st != CPE_OK:
        raise CpeError(st, "cpe_rows8_unpack")
    return x


class RmsNorm:
    """Handle of one RMS norm (channels, dtype) for calls of up to ``max_rows``
    rows.  Matrices are [rows][channels] tensors with contiguous channels and
    any row stride."""
    _device = None      # the handle's; a host tensor's get_device() is -1

    def __init__(self, max_rows: int, channels: int, dtype: str, eps: float = 1e-6):
        self.channels, self.dtype = _int32(channels, "channels"), dtype
        self.eps, self._torch_dtype, self._lib = float(eps), torch_dtype(dtype), library()
        h = ctypes.c_void_p()
        st = self._lib.cpe_rms_create(ctypes.byref(h), _int32(max_rows, "max_rows"), self.channels, DTYPES[dtype],
                                      self.eps)
        if st != CPE_OK:
            raise CpeError(st, "cpe_rms_create")
        self._h, self._device = h, torch.cuda.current_device()

    def _matrix(self, t, rows, name: str):
        return _matrix(t, rows, self.channels, name, self._device, self._torch_dtype)

    def forward(self, x, gamma, residual=None, sum=None, y=None, q=None, scale=None, rstd=None, stream=None) -> int:
        """cpe_rms_forward: writes those of sum, y, (q, scale) and rstd that
        are given."""
        rows, dev = x.shape[0], self._device
        if rows >> 31:
            raise ValueError(f"x: {rows} is no 32-bit number of rows")
        px, x_ld = self._matrix(x, None, "x")
        pr, r_ld = self._matrix(residual, rows, "residual")
        ph, h_ld = self._matrix(sum, rows, "sum")
        py, y_ld = self._matrix(y, rows, "y")
        pq, q_ld = _matrix(q, rows, self.channels, "q", dev, torch.int8)
        return self._lib.cpe_rms_forward(self._h, _stream(stream, dev), rows, px, x_ld, pr, r_ld,
                                         _vector(gamma, self.channels, "gamma", dev), ph, h_ld, py, y_ld, pq, q_ld,
                                         _vector(scale, rows, "scale", dev), _vector(rstd, rows, "rstd", dev))

    def backward(self, h, dy, gamma, rstd, dx=None, dgamma=None, dsum=None, h_scale=None, stream=None) -> int:
        """cpe_rms_backward: writes those of dx and dgamma that are given.
        ``h`` is the forward's sum (or its x, without a residual), or that in
        8 bits with ``h_scale``."""
        rows, dev = h.shape[0], self._device
        if rows >> 31:
            raise ValueError(f"h: {rows} is no 32-bit number of rows")
        ph, h_ld = _matrix(h, None, self.channels, "h", dev, self._torch_dtype if h_scale is None else torch.int8)
        pd, d_ld = self._matrix(dy, rows, "dy")
        ps, s_ld = self._matrix(dsum, rows, "dsum")
        po, o_ld = self._matrix(dx, rows, "dx")
        return self._lib.cpe_rms_backward(self._h, _stream(stream, dev), rows, ph, h_ld,
                                          _vector(h_scale, rows, "h_scale", dev), pd, d_ld,
                                          _vector(gamma, self.channels, "gamma", dev),
                                          _vector(rstd, rows, "rstd", dev), ps, s_ld, po, o_ld,
                                          _vector(dgamma, self.channels, "dgamma", dev))

    def run(self, x, gamma, residual=None, packed=False, stream=None):
        """forward into new tensors: (y, rstd), or ((q, scale), rstd) where
        ``packed``; with a residual the sum comes first.  Not recorded by
        autograd: tensors that require a gradient are refused while it records."""
        _unrecorded("RmsNorm.run", x, gamma, residual)
        with _allocating(stream):
            rstd = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
            total = None if residual is None else torch.empty(x.shape, dtype=x.dtype, device=x.device)
            y = None if packed else torch.empty(x.shape, dtype=x.dtype, device=x.device)
            q, scale = (torch.empty(x.shape, dtype=torch.int8, device=x.device),
                        torch.empty(x.shape[0], dtype=torch.float32, device=x.device)) if packed else (None, None)
        st = self.forward(x, gamma, residual, total, y, q, scale, rstd, stream)
        if st != CPE_OK:
            raise CpeError(st, "cpe_rms_forward")
        out = ((q, scale) if packed else y, rstd)
        return out if residual is None else (total, *out)

    def run_backward(self, h, dy, gamma, rstd, dsum=None, h_scale=None, stream=None):
        """backward into new tensors: (dx, dgamma)."""
        with _allocating(stream):
            dx = torch.empty(dy.shape, dtype=dy.dtype, device=dy.device)
            dgamma = torch.empty(self.channels, dtype=torch.float32, device=dy.device)
        st = self.backward(h, dy, gamma, rstd, dx, dgamma, dsum, h_scale, stream)
        if st != CPE_OK:
            raise CpeError(st, "cpe_rms_backward")
        return dx, dgamma

    def workspace_bytes(self) -> int:
        return int(self._lib.cpe_rms_workspace_bytes(self._h))

    def close(self):
        if getattr(self, "_h", None):
            self._lib.cpe_rms_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Linear8:
    """Handle of one integer matrix product (features, dtype of the output,
    activation) for calls of up to ``max_rows`` rows.  The weight is in 8 bits
    as well, [out][in] with a scale for each output feature: ``packed(weight)``."""
    _device = None      # the handle's; a host tensor's get_device() is -1

    def __init__(self, max_rows: int, in_features: int, out_features: int, dtype: str, activation: str = "none"):
        self.in_features, self.out_features = _int32(in_features, "in_features"), _int32(out_features, "out_features")
        self.dtype = dtype
        self._torch_dtype, self._lib = torch_dtype(dtype), library()
        h = ctypes.c_void_p()
        st = self._lib.cpe_linear8_create(ctypes.byref(h), _int32(max_rows, "max_rows"), self.in_features,
                                          self.out_features, DTYPES[dtype], ACTIVATIONS[activation])
        if st != CPE_OK:
            raise CpeError(st, "cpe_linear8_create")
        self._h, self._device = h, torch.cuda.current_device()

    def forward(self, q, scale, weight, weight_scale, bias, y, residual=None, preact=None, stream=None) -> int:
        """cpe_linear8_forward: ``preact`` receives the value before the
        activation, which the gradient needs."""
        rows, n, dev = q.shape[0], self.out_features, self._device
        if rows >> 31:
            raise ValueError(f"q: {rows} is no 32-bit number of rows")
        pq, q_ld, ps = _packed(q, scale, None, self.in_features, "q", dev)
        pw, w_ld, pt = _packed(weight, weight_scale, n, self.in_features, "weight", dev)
        py, y_ld = _matrix(y, rows, n, "y", dev, self._torch_dtype)
        pr, r_ld = _matrix(residual, rows, n, "residual", dev, self._torch_dtype)
        pz, z_ld = _matrix(preact, rows, n, "preact", dev, self._torch_dtype)
        return self._lib.cpe_linear8_forward(self._h, _stream(stream, dev), rows, pq, q_ld, ps, pw, w_ld, pt,
                                             _vector(bias, n, "bias", dev), pr, r_ld, py, y_ld, pz, z_ld)

    def run(self, q, scale, weight, weight_scale, bias=None, residual=None, keep=False, stream=None):
        """forward into new tensors: y, or (y, preact) where ``keep``.  Not
        recorded by autograd: tensors that require a gradient are refused while
        it records."""
        _unrecorded("Linear8.run", scale, weight_scale, bias, residual)
        with _allocating(stream):
            y = torch.empty((q.shape[0], self.out_features), dtype=self._torch_dtype, device=q.device)
            preact = torch.empty_like(y) if keep else None
        st = self.forward(q, scale, weight, weight_scale, bias, y, residual, preact, stream)
        if st != CPE_OK:
            raise CpeError(st, "cpe_linear8_forward")
        return (y, preact) if keep else y

    def workspace_bytes(self) -> int:
        return int(self._lib.cpe_linear8_workspace_bytes(self._h))

    def close(self):
        if getattr(self, "_h", None):
            self._lib.cpe_linear8_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
