"""The head operators' entry points refuse bad arguments on the host (no GPU
work is issued), and the binding refuses what the C ABI cannot see."""
import ctypes

import pytest

from paper_2609_16874_amd import native

torch = pytest.importorskip("torch")


def _handle():
    return ctypes.c_void_p(123)


@pytest.mark.parametrize("change", [dict(samples=0), dict(samples=65536), dict(pixels=0), dict(pixels=2 ** 31 - 1),
                                    dict(channels=0), dict(channels=8193), dict(groups=0), dict(groups=3),
                                    dict(dtype=3), dict(dtype=-1), dict(act=4), dict(act=-1), dict(eps=0.0),
                                    dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))])
def test_norm_create_refuses(change):
    a = dict(samples=2, pixels=16, channels=8, groups=2, dtype=1, act=2, eps=1e-5)
    a.update(change)
    h = _handle()
    assert native.library().cpe_norm_create(ctypes.byref(h), *a.values()) == native.CPE_ERR_INVALID_ARG
    assert h.value is None


@pytest.mark.parametrize("change", [dict(rows=0), dict(rows=2 ** 31 - 1), dict(k=0), dict(k=65537), dict(n=0),
                                    dict(n=65537), dict(dtype=3), dict(act=4), dict(act=-1)])
def test_linear_create_refuses(change):
    a = dict(rows=16, k=8, n=2, dtype=1, act=2)
    a.update(change)
    h = _handle()
    assert native.library().cpe_linear_create(ctypes.byref(h), *a.values()) == native.CPE_ERR_INVALID_ARG
    assert h.value is None


def test_null_handles():
    lib, bad = native.library(), native.CPE_ERR_INVALID_ARG
    assert lib.cpe_norm_create(None, 1, 1, 8, 2, 0, 0, 1e-5) == bad
    assert lib.cpe_linear_create(None, 1, 8, 8, 0, 0) == bad
    assert lib.cpe_norm_forward(None, None, 0, 0, None, 0, 0, None, None, None, None, 0, 0, None) == bad
    assert lib.cpe_norm_backward(None, None, 0, 0, None, 0, 0, None, 0, 0, None, None, None, None, None, 0, 0, None,
                                 None) == bad
    assert lib.cpe_linear_forward(None, None, 0, None, 0, None, 0, None, None, 0, None, 0, None, 0) == bad
    assert lib.cpe_linear_backward(None, None, 0, None, 0, None, 0, None, 0, None, 0, None, 0, None, 0, None) == bad
    assert lib.cpe_norm_destroy(None) == 0 and lib.cpe_linear_destroy(None) == 0
    assert lib.cpe_norm_workspace_bytes(None) == 0 and lib.cpe_linear_workspace_bytes(None) == 0


def test_the_decoder_takes_no_bf16():
    import numpy as np
    h, f = _handle(), np.ones(4)
    assert native.library().cpe_decode_create(ctypes.byref(h), 16, 16, 16, 2, f.ctypes.data,
                                              f.ctypes.data, 4, 8, 8, 16) == native.CPE_ERR_INVALID_ARG


def _norm_call(h, lib, **change):
    """A forward call whose pointers are never followed unless it is accepted."""
    a = dict(samples=2, pixels=4, x=4096, x_ld=8, x_sample=32, gamma=None, beta=None, valid=None, y=8192, y_ld=8,
             y_sample=32, stats=None)
    a.update(change)
    return lib.cpe_norm_forward(h, None, *a.values())


def _linear_call(h, lib, **change):
    a = dict(rows=4, x=4096, x_ld=8, w=8192, w_ld=8, bias=None, residual=None, residual_ld=0, y=12288, y_ld=6,
             preact=None, preact_ld=0)
    a.update(change)
    return lib.cpe_linear_forward(h, None, *a.values())


@pytest.mark.gpu
@pytest.mark.parametrize("change", [dict(samples=3), dict(samples=-1), dict(pixels=5), dict(pixels=-1), dict(x=None),
                                    dict(y=None), dict(x=4097), dict(y=8193), dict(x_ld=7), dict(x_ld=-8),
                                    dict(y_ld=7), dict(x_sample=31), dict(x_sample=-32), dict(y_sample=31),
                                    dict(x_ld=2 ** 41), dict(gamma=4098), dict(beta=4097), dict(valid=4098),
                                    dict(stats=4100), dict(y=4096, y_ld=9, y_sample=36)])
def test_norm_forward_refuses(change):
    lib, h = native.library(), ctypes.c_void_p()
    assert lib.cpe_norm_create(ctypes.byref(h), 2, 4, 8, 2, 1, 0, 1e-5) == 0
    assert _norm_call(h, lib, **change) == native.CPE_ERR_INVALID_ARG
    assert lib.cpe_norm_destroy(h) == 0


@pytest.mark.gpu
def test_norm_backward_refuses():
    lib, h, bad = native.library(), ctypes.c_void_p(), native.CPE_ERR_INVALID_ARG
    assert lib.cpe_norm_create(ctypes.byref(h), 2, 4, 8, 2, 1, 0, 1e-5) == 0
    good = dict(samples=2, pixels=4, x=4096, x_ld=8, x_sample=32, dy=8192, dy_ld=8, dy_sample=32, gamma=None,
                beta=None, valid=None, stats=16384, dx=12288, dx_ld=8, dx_sample=32, dgamma=None, dbeta=None)
    for change in (dict(dx=None), dict(stats=None), dict(stats=16388), dict(dy=None), dict(dy_ld=7), dict(dx_ld=7),
                   dict(dx=4097), dict(dgamma=4098), dict(dbeta=4097), dict(samples=3), dict(pixels=5),
                   dict(dx=8192, dx_ld=9, dx_sample=36), dict(dx=4096, dx_ld=9, dx_sample=36), dict(dy_sample=31)):
        assert lib.cpe_norm_backward(h, None, *{**good, **change}.values()) == bad, change
    assert lib.cpe_norm_destroy(h) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("change", [dict(rows=5), dict(rows=-1), dict(x=None), dict(w=None), dict(y=None),
                                    dict(x=4097), dict(x_ld=7), dict(w_ld=7), dict(y_ld=5), dict(bias=4098),
                                    dict(residual=16384, residual_ld=5), dict(residual=16385, residual_ld=6),
                                    dict(residual=12288, residual_ld=7), dict(preact=16384, preact_ld=5),
                                    dict(preact=12288, preact_ld=6)])
def test_linear_forward_refuses(change):
    lib, h = native.library(), ctypes.c_void_p()
    assert lib.cpe_linear_create(ctypes.byref(h), 4, 8, 6, 1, 0) == 0
    assert _linear_call(h, lib, **change) == native.CPE_ERR_INVALID_ARG
    assert lib.cpe_linear_destroy(h) == 0


@pytest.mark.gpu
def test_linear_backward_refuses():
    lib, h, bad = native.library(), ctypes.c_void_p(), native.CPE_ERR_INVALID_ARG
    assert lib.cpe_linear_create(ctypes.byref(h), 4, 8, 6, 1, 2) == 0
    good = dict(rows=4, x=4096, x_ld=8, w=8192, w_ld=8, dy=12288, dy_ld=6, preact=16384, preact_ld=6, dx=20480,
                dx_ld=8, dw=24576, dw_ld=8, dbias=28672)
    for change in (dict(dx=None, dw=None, dbias=None), dict(preact=None), dict(preact_ld=5), dict(dy=None),
                   dict(dy_ld=5), dict(x=None), dict(w=None), dict(dx_ld=7), dict(dw_ld=7), dict(dbias=28674),
                   dict(dx=4096), dict(dx=12288), dict(dw=8192), dict(dw=20480), dict(rows=5), dict(rows=-1),
                   dict(dw=24577)):
        assert lib.cpe_linear_backward(h, None, *{**good, **change}.values()) == bad, change
    assert lib.cpe_linear_destroy(h) == 0


def test_binding_refuses_what_the_abi_cannot_see():
    from paper_2609_16874_amd import head
    with pytest.raises(KeyError):
        head.GroupNorm(1, 1, 8, 2, "f64")
    with pytest.raises(KeyError):
        head.Linear(1, 8, 8, "f16", "tanh")
    n, lin = object.__new__(head.GroupNorm), object.__new__(head.Linear)
    n.channels, n.groups, n._torch_dtype = 8, 2, torch.float16
    lin.in_features, lin.out_features, lin._torch_dtype = 8, 6, torch.float16
    x = torch.zeros((2, 4, 8), dtype=torch.float16)
    with pytest.raises(ValueError):       # host memory
        n.forward(x, None, None, x)
    with pytest.raises(ValueError):
        n.forward(x[0, 0], None, None, x)
    with pytest.raises(ValueError):
        lin.forward(x[0], x[0, :6], None, x[0])


@pytest.mark.gpu
@pytest.mark.parametrize("change", [dict(y=4096), dict(y=8192), dict(preact=4096, preact_ld=8),
                                    dict(preact=8192, preact_ld=8), dict(preact=12288, preact_ld=8),
                                    dict(preact=16384, preact_ld=8, residual=16384, residual_ld=8)])
def test_linear_forward_refuses_outputs_in_place_of_inputs(change):
    """Equal features, so that the shapes alone would allow it."""
    lib, h = native.library(), ctypes.c_void_p()
    assert lib.cpe_linear_create(ctypes.byref(h), 4, 8, 8, 1, 0) == 0
    assert _linear_call(h, lib, y_ld=8, **change) == native.CPE_ERR_INVALID_ARG
    assert lib.cpe_linear_destroy(h) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("pixels", [2 ** 23 + 1, 2 ** 24 + 1, 2 ** 31 - 2 ** 23])
@pytest.mark.parametrize("sample", [-2 ** 62, -32, 0, 7, 2 ** 40 - 7, 2 ** 40, 2 ** 40 + 1])
def test_norm_strides_whose_product_passes_64_bits(pixels, sample):
    """Pixel strides of 2^40: no sample stride keeps two such samples apart."""
    lib, h = native.library(), ctypes.c_void_p()
    assert lib.cpe_norm_create(ctypes.byref(h), 2, 2 ** 31 - 2 ** 23, 8, 2, 1, 0, 1e-5) == 0
    far = dict(pixels=pixels, x_ld=2 ** 40, x_sample=sample)
    assert _norm_call(h, lib, **far) == native.CPE_ERR_INVALID_ARG
    assert _norm_call(h, lib, pixels=pixels, x_ld=8, x_sample=8 * pixels, y_ld=2 ** 40,
                      y_sample=sample) == native.CPE_ERR_INVALID_ARG
    assert lib.cpe_norm_destroy(h) == 0
