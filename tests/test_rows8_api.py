"""The entry points on rows in 8 bits refuse bad arguments on the host (no GPU
work is issued), and the binding refuses what the C ABI cannot see."""
import ctypes

import pytest

from paper_2609_16874_amd import native
from tests.test_head_binding import Recorder, Stream, Tensor

torch = pytest.importorskip("torch")
BAD = native.CPE_ERR_INVALID_ARG
I8, F32 = torch.int8, torch.float32


@pytest.mark.parametrize("change", [dict(rows=-1), dict(rows=2 ** 31 - 1), dict(width=0), dict(width=65537),
                                    dict(dtype=3), dict(dtype=-1), dict(x=None), dict(x=4097), dict(x_ld=7),
                                    dict(x_ld=-8), dict(x_ld=2 ** 41), dict(q=None), dict(q_ld=7), dict(q_ld=2 ** 41),
                                    dict(scale=None), dict(scale=12290), dict(q=4096), dict(scale=4096),
                                    dict(scale=8192)])
def test_pack_and_unpack_refuse(change):
    """(The pointers are never followed: every call is refused.)"""
    a = dict(rows=4, width=8, dtype=1, x=4096, x_ld=8, q=8192, q_ld=8, scale=12288)
    a.update(change)
    lib = native.library()
    assert lib.cpe_rows8_pack(None, *a.values()) == BAD
    if change != dict(scale=8192):
        assert lib.cpe_rows8_unpack(None, a["rows"], a["width"], a["q"], a["q_ld"], a["scale"], a["dtype"], a["x"],
                                    a["x_ld"]) == BAD


def test_no_rows_need_no_pointers():
    lib = native.library()
    assert lib.cpe_rows8_pack(None, 0, 8, 1, None, 0, None, 0, None) == 0
    assert lib.cpe_rows8_unpack(None, 0, 8, None, 0, None, 1, None, 0) == 0


@pytest.mark.parametrize("change", [dict(rows=0), dict(rows=2 ** 31 - 1), dict(channels=0), dict(channels=16385),
                                    dict(dtype=3), dict(dtype=-1), dict(eps=0.0), dict(eps=-1.0), dict(eps=1e-39),
                                    dict(eps=float("nan")), dict(eps=float("inf"))])
def test_rms_create_refuses(change):
    a = dict(rows=16, channels=8, dtype=1, eps=1e-6)
    a.update(change)
    h = ctypes.c_void_p(123)
    assert native.library().cpe_rms_create(ctypes.byref(h), *a.values()) == BAD
    assert h.value is None


@pytest.mark.parametrize("change", [dict(rows=0), dict(rows=2 ** 31 - 1), dict(k=0), dict(k=65537), dict(n=0),
                                    dict(n=65537), dict(dtype=3), dict(act=4), dict(act=-1)])
def test_linear8_create_refuses(change):
    a = dict(rows=16, k=8, n=2, dtype=1, act=2)
    a.update(change)
    h = ctypes.c_void_p(123)
    assert native.library().cpe_linear8_create(ctypes.byref(h), *a.values()) == BAD
    assert h.value is None


def test_null_handles():
    lib = native.library()
    assert lib.cpe_rms_create(None, 1, 8, 0, 1e-6) == BAD and lib.cpe_linear8_create(None, 1, 8, 8, 0, 0) == BAD
    assert lib.cpe_rms_forward(None, None, 0, *[None, 0] * 2, None, *[None, 0] * 3, None, None) == BAD
    assert lib.cpe_rms_backward(None, None, 0, None, 0, None, None, 0, None, None, None, 0, None, 0, None) == BAD
    assert lib.cpe_linear8_forward(None, None, 0, None, 0, None, None, 0, None, None, None, 0, None, 0, None, 0) == BAD
    assert lib.cpe_linear_backward8(None, None, 0, None, 0, None, None, 0, None, 0, None, 0, None, None, 0, None, 0,
                                    None) == BAD
    assert lib.cpe_rms_destroy(None) == 0 and lib.cpe_linear8_destroy(None) == 0
    assert lib.cpe_rms_workspace_bytes(None) == 0 and lib.cpe_linear8_workspace_bytes(None) == 0


@pytest.mark.gpu
def test_rms_calls_refuse():
    lib, h = native.library(), ctypes.c_void_p()
    assert lib.cpe_rms_create(ctypes.byref(h), 4, 8, 1, 1e-6) == 0
    good = dict(rows=4, x=4096, x_ld=8, residual=8192, residual_ld=8, gamma=None, sum=12288, sum_ld=8, y=16384, y_ld=8,
                q=20480, q_ld=8, scale=24576, rstd=28672)
    for change in (dict(rows=5), dict(rows=-1), dict(x=None), dict(x=4097), dict(x_ld=7), dict(residual=8193),
                   dict(residual_ld=7), dict(gamma=2), dict(sum=12289), dict(sum_ld=7), dict(y=16385), dict(y_ld=-8),
                   dict(q_ld=7), dict(q=None), dict(scale=None), dict(scale=24578), dict(rstd=28674), dict(y=12288),
                   dict(sum=4096, sum_ld=9), dict(sum=8192, sum_ld=9), dict(y=4096, y_ld=9), dict(y=8192, y_ld=9),
                   dict(q=4096), dict(q=8192), dict(q=12288), dict(q=16384), dict(x_ld=2 ** 41), dict(rstd=24576),
                   dict(sum=None, y=None, q=None, scale=None)):
        assert lib.cpe_rms_forward(h, None, *{**good, **change}.values()) == BAD, change
    good = dict(rows=4, h=4096, h_ld=8, h_scale=None, dy=8192, dy_ld=8, gamma=None, rstd=12288, dsum=16384, dsum_ld=8,
                dx=20480, dx_ld=8, dgamma=24576)
    for change in (dict(rows=5), dict(rows=-1), dict(h=None), dict(h=4097), dict(h_ld=7), dict(h_scale=2), dict(dy=None),
                   dict(dy=8193), dict(dy_ld=7), dict(gamma=2), dict(rstd=None), dict(rstd=12290), dict(dsum=16385),
                   dict(dsum_ld=7), dict(dx=20481), dict(dx_ld=7), dict(dgamma=24578), dict(dx=None, dgamma=None),
                   dict(dx=4096, dx_ld=9), dict(dx=8192, dx_ld=9), dict(dx=16384, dx_ld=9),
                   dict(dx=4096, h_scale=28672), dict(h_ld=7, h_scale=28672)):
        assert lib.cpe_rms_backward(h, None, *{**good, **change}.values()) == BAD, change
    assert lib.cpe_rms_destroy(h) == 0


@pytest.mark.gpu
def test_linear8_calls_refuse():
    lib, h = native.library(), ctypes.c_void_p()
    assert lib.cpe_linear8_create(ctypes.byref(h), 4, 8, 8, 1, 2) == 0
    good = dict(rows=4, q=4096, q_ld=8, scale=8192, w=12288, w_ld=8, w_scale=16384, bias=None, residual=20480,
                residual_ld=8, y=24576, y_ld=8, preact=28672, preact_ld=8)
    for change in (dict(rows=5), dict(rows=-1), dict(q=None), dict(q_ld=7), dict(scale=None), dict(scale=2), dict(w=None),
                   dict(w_ld=7), dict(w_scale=None), dict(w_scale=2), dict(bias=2), dict(residual=20481),
                   dict(residual_ld=7), dict(y=None), dict(y=24577), dict(y_ld=7), dict(preact=28673),
                   dict(preact_ld=7), dict(y=4096), dict(y=12288), dict(preact=24576), dict(preact=20480),
                   dict(preact=4096), dict(preact=12288), dict(residual=24576, residual_ld=9)):
        assert lib.cpe_linear8_forward(h, None, *{**good, **change}.values()) == BAD, change
    assert lib.cpe_linear8_destroy(h) == 0
    h = ctypes.c_void_p()
    assert lib.cpe_linear_create(ctypes.byref(h), 4, 8, 6, 1, 2) == 0
    good = dict(rows=4, q=4096, q_ld=8, scale=8192, w=12288, w_ld=8, dy=16384, dy_ld=6, zq=20480, zq_ld=6,
                z_scale=24576, dx=28672, dx_ld=8, dw=32768, dw_ld=8, dbias=36864)
    for change in (dict(rows=5), dict(rows=-1), dict(q=None), dict(q_ld=7), dict(scale=None), dict(scale=2), dict(w=None),
                   dict(w_ld=7), dict(dy=None), dict(dy_ld=5), dict(zq=None), dict(zq_ld=5), dict(z_scale=None),
                   dict(z_scale=2), dict(dx_ld=7), dict(dx=28673), dict(dw_ld=7), dict(dw=32769), dict(dbias=2),
                   dict(dx=None, dw=None, dbias=None), dict(dx=4096), dict(dx=12288), dict(dx=16384), dict(dx=20480),
                   dict(dw=4096), dict(dw=12288), dict(dw=16384), dict(dw=20480), dict(dw=28672)):
        assert lib.cpe_linear_backward8(h, None, *{**good, **change}.values()) == BAD, change
    assert lib.cpe_linear_destroy(h) == 0


# -- the binding, with a recorder in the library's place --------------------------

def _rms(channels=8):
    from paper_2609_16874_amd import rows8
    h = object.__new__(rows8.RmsNorm)
    h.channels, h.dtype, h.eps, h._torch_dtype, h._lib, h._h, h._device = channels, "f16", 1e-6, torch.float16, \
        Recorder(), 123, 0
    return h


def _linear8(k=8, n=6):
    from paper_2609_16874_amd import rows8
    h = object.__new__(rows8.Linear8)
    h.in_features, h.out_features, h.dtype = k, n, "f16"
    h._torch_dtype, h._lib, h._h, h._device = torch.float16, Recorder(), 123, 0
    return h


def _linear(k=8, n=6):
    from paper_2609_16874_amd import head
    h = object.__new__(head.Linear)
    h.in_features, h.out_features, h.dtype = k, n, "f16"
    h._torch_dtype, h._lib, h._h, h._device = torch.float16, Recorder(), 123, 0
    return h


@pytest.fixture
def recorded(monkeypatch):
    from paper_2609_16874_amd import head, rows8
    lib = Recorder()
    monkeypatch.setattr(rows8, "library", lambda: lib)
    monkeypatch.setattr(rows8, "_current_device", lambda: 0)
    for m in (head, rows8):
        monkeypatch.setattr(m, "_stream", lambda stream, device: 0 if stream is None else stream.cuda_stream)
    return lib


def test_what_the_calls_pass_on(recorded):
    """Pointers, strides and sizes, in the header's order."""
    from paper_2609_16874_amd import rows8
    x, q, s = Tensor((4, 8), strides=(10, 1), pointer=16), Tensor((4, 8), I8, (24, 1), pointer=32), Tensor((4,), F32)
    assert rows8.pack(x, q, s, Stream()) == 0 and rows8.unpack(q, s, x) == 0
    assert recorded.calls == [("cpe_rows8_pack", (77, 4, 8, 1, 16, 10, 32, 24, 4096)),
                              ("cpe_rows8_unpack", (0, 4, 8, 32, 24, 4096, 1, 16, 10))]
    r = _rms()
    assert r.forward(x, None, residual=x, sum=x, y=x, q=q, scale=s, rstd=s) == 0
    assert r._lib.calls == [("cpe_rms_forward", (123, 0, 4, 16, 10, 16, 10, None, 16, 10, 16, 10, 32, 24, 4096, 4096))]
    r = _rms()
    assert r.backward(q, x, None, s, dx=x, h_scale=s) == 0
    assert r._lib.calls == [("cpe_rms_backward", (123, 0, 4, 32, 24, 4096, 16, 10, None, 4096, None, 0, 16, 10, None))]
    w, t, y = Tensor((6, 8), I8, pointer=48), Tensor((6,), F32, pointer=64), Tensor((4, 6), pointer=80)
    f = _linear8()
    assert f.forward(q, s, w, t, t, y, residual=y, preact=y) == 0
    assert f._lib.calls == [("cpe_linear8_forward", (123, 0, 4, 32, 24, 4096, 48, 8, 64, 64, 80, 6, 80, 6, 80, 6))]
    b = _linear()
    wd, zq = Tensor((6, 8), pointer=96), Tensor((4, 6), I8, pointer=112)
    assert b.backward8(q, s, wd, y, zq, s, dx=x, dweight=wd, dbias=t) == 0
    assert b._lib.calls == [("cpe_linear_backward8", (123, 0, 4, 32, 24, 4096, 96, 8, 80, 6, 112, 6, 4096, 16, 10, 96, 8,
                                                      64))]


def test_binding_refuses_what_the_abi_cannot_see(recorded):
    from paper_2609_16874_amd import rows8
    x, q, s = Tensor((4, 8)), Tensor((4, 8), I8), Tensor((4,), F32)
    for bad in (dict(x=Tensor((4, 8), torch.float64)), dict(x=Tensor((4, 9))), dict(x=Tensor((5, 8))), dict(q=x),
                dict(q=Tensor((4, 8), torch.uint8)), dict(s=Tensor((4,))), dict(s=Tensor((5,), F32)),
                dict(s=Tensor((4,), F32, device=1)), dict(q=Tensor((4, 8), I8, (1, 4))), dict(x=Tensor((4, 8, 1))),
                dict(x=Tensor((4, 8), device=1)), dict(q=Tensor((2 ** 31, 8), I8))):
        a = dict(x=x, q=q, s=s, **{})
        a.update(bad)
        with pytest.raises(ValueError):
            rows8.pack(a["x"], a["q"], a["s"])
        with pytest.raises(ValueError):
            rows8.unpack(a["q"], a["s"], a["x"])
    assert recorded.calls == []
    r = _rms()
    for bad in (dict(x=Tensor((4, 9))), dict(x=Tensor((4, 8), F32)), dict(residual=Tensor((5, 8))), dict(sum=q),
                dict(y=Tensor((4, 8), device=1)), dict(q=x), dict(scale=x), dict(rstd=Tensor((8,), F32)),
                dict(gamma=Tensor((4,), F32))):
        a = dict(x=x, gamma=None, residual=x, sum=x, y=x, q=q, scale=s, rstd=s)
        a.update(bad)
        with pytest.raises(ValueError):
            r.forward(**a)
    for bad in (dict(h=x), dict(h=q, h_scale=None), dict(dy=q), dict(rstd=None, dsum=Tensor((3, 8))),
                dict(dx=Tensor((4, 8), F32)), dict(dgamma=Tensor((4,), F32)), dict(h_scale=Tensor((8,), F32))):
        a = dict(h=q, dy=x, gamma=None, rstd=s, dx=x, dgamma=None, dsum=None, h_scale=s)
        a.update(bad)
        with pytest.raises(ValueError):
            r.backward(**a)
    assert r._lib.calls == []
    w, t, y = Tensor((6, 8), I8), Tensor((6,), F32), Tensor((4, 6))
    f = _linear8()
    for bad in (dict(q=x), dict(scale=t), dict(weight=Tensor((6, 8))), dict(weight=Tensor((5, 8), I8)),
                dict(weight_scale=s), dict(bias=s), dict(y=Tensor((4, 6), F32)), dict(residual=Tensor((4, 7))),
                dict(preact=Tensor((3, 6))), dict(q=Tensor((2 ** 31, 8), I8))):
        a = dict(q=q, scale=s, weight=w, weight_scale=t, bias=None, y=y, residual=None, preact=None)
        a.update(bad)
        with pytest.raises(ValueError):
            f.forward(**a)
    b = _linear()
    for bad in (dict(q=x), dict(scale=t), dict(weight=w), dict(dy=Tensor((4, 6), I8)), dict(preact_q=y),
                dict(preact_scale=t), dict(dx=q), dict(dweight=w), dict(dbias=s)):
        a = dict(q=q, scale=s, weight=Tensor((6, 8)), dy=y, preact_q=Tensor((4, 6), I8), preact_scale=s, dx=None,
                 dweight=None, dbias=t)
        a.update(bad)
        with pytest.raises(ValueError):
            b.backward8(**a)
    assert f._lib.calls == [] and b._lib.calls == []


def test_runs_are_not_recorded_by_autograd(recorded):
    from paper_2609_16874_amd import rows8
    x, s = Tensor((4, 8)), Tensor((4,), F32)
    x.requires_grad = True
    for call in (lambda: rows8.packed(x), lambda: _rms().run(x, None),
                 lambda: _linear8().run(Tensor((4, 8), I8), s, Tensor((6, 8), I8), Tensor((6,), F32), residual=x)):
        with pytest.raises(ValueError, match="autograd"):
            call()


@pytest.mark.parametrize("given", [True, False])
def test_outputs_are_allocated_on_the_stream_that_writes_them(given, recorded, monkeypatch):
    import contextlib
    from paper_2609_16874_amd import head, rows8
    inside, streams = [], []

    @contextlib.contextmanager
    def on(stream):
        streams.append(stream)
        yield
        streams.pop()

    def empty(shape, dtype=None, device=None):
        inside.append(streams[-1] if streams else None)
        return Tensor((shape,) if isinstance(shape, int) else shape, dtype)

    monkeypatch.setattr(head.torch.cuda, "stream", on)
    monkeypatch.setattr(head.torch, "empty", empty)
    monkeypatch.setattr(head.torch, "empty_like", lambda t: empty(t.shape, t.dtype))
    stream = Stream() if given else None
    x, q, s, y = Tensor((4, 8)), Tensor((4, 8), I8), Tensor((4,), F32), Tensor((4, 6))
    rows8.packed(x, stream)
    rows8.unpacked(q, s, "bf16", stream)
    _rms().run(x, None, x, packed=True, stream=stream)
    _rms().run_backward(q, x, None, s, h_scale=s, stream=stream)
    _linear8().run(q, s, Tensor((6, 8), I8), Tensor((6,), F32), keep=True, stream=stream)
    _linear().run_backward8(q, s, Tensor((6, 8)), y, Tensor((4, 6), I8), s, stream=stream)
    assert len(inside) == 14 and all(t is stream for t in inside)


@pytest.mark.parametrize("which", ["x", "residual", "gamma"])
def test_a_block_that_would_lose_a_gradient_refuses(which):
    """(The norm writes into tensors of the block's own, which no autograd sees.)"""
    from paper_2609_16874_amd.pixel_block import PixelBlock
    t = {k: torch.zeros((4, 8) if k != "gamma" else 8, requires_grad=k == which) for k in ("x", "residual", "gamma")}
    b = object.__new__(PixelBlock)
    b.params, b.checkpoint8, b.norm = {"gamma": t["gamma"]}, False, _rms()
    with pytest.raises(ValueError, match="autograd"):
        b.forward(t["x"], t["residual"])
    assert b.norm._lib.calls == []
