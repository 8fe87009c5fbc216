"""The host side of the operators on rows in 8 bits, compiled without kernels and
with a runtime that only counts launches: calls whose outputs are an input or
another output are refused before anything is launched, and the calls that the
header allows are not."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2609_16874_amd import build

BAD = 1
STUB = r"""
#include <cstdlib>
#include "head/linear.hpp"
#include "rows8/linear8.hpp"
#include "rows8/rows.hpp"
int launched = 0;
extern "C" {
int launches() { return launched; }
hipError_t hipGetDevice(int *d) { *d = 0; return hipSuccess; }
hipError_t hipMalloc(void **p, size_t n) { *p = malloc(n); return *p ? hipSuccess : hipErrorOutOfMemory; }
hipError_t hipFree(void *p) { free(p); return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
}
namespace cpe {
#define NONE(name, ...) hipError_t name(__VA_ARGS__, hipStream_t) { launched++; return hipSuccess; }
#define TYPE(t)                                                                                          \
    NONE(launch_pack_##t, const RowsArgs &) NONE(launch_unpack_##t, const UnpackArgs &)                   \
    NONE(launch_rms_##t, const RowsArgs &) NONE(launch_rms_grad_##t, RmsGradArgs)                         \
    NONE(launch_gemm8_##t, const Gemm8Args &) NONE(launch_gemm_##t, const GemmArgs &)                     \
    NONE(launch_grad_##t, const GradArgs &) NONE(launch_rows_grad_##t, const WholeGradArgs &)
TYPE(f32) TYPE(f16) TYPE(bf16)
NONE(launch_narrow_grad_f16, WholeGradArgs) NONE(launch_narrow_grad_bf16, WholeGradArgs)
}
"""

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    folder = tmp_path_factory.mktemp("host")
    (folder / "stub.hip").write_text(STUB)
    out = folder / "libhost.so"
    sources = [os.path.join(build.CSRC, *p) for p in (("rows8", "rows8.hip"), ("rows8", "linear8.hip"),
                                                      ("head", "linear.hip"))]
    objects = []
    for i, s in enumerate([*sources, str(folder / "stub.hip")]):
        objects.append(str(folder / f"{i}.o"))
        subprocess.run(["hipcc", "--offload-arch=gfx950", "--cuda-host-only", "-O1", "-std=c++17", "-fPIC", "-I",
                        build.INCLUDE, "-I", build.CSRC, "-c", "-o", objects[-1], s], check=True, capture_output=True)
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", "-o", str(out), *objects], check=True, capture_output=True)
    h = ctypes.CDLL(str(out))
    P, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    h.cpe_rms_create.argtypes = [ctypes.POINTER(P), i32, i32, i32, ctypes.c_float]
    h.cpe_rms_forward.argtypes = [P, P, i32, P, i64, P, i64, P, P, i64, P, i64, P, i64, P, P]
    h.cpe_rms_backward.argtypes = [P, P, i32, P, i64, P, P, i64, P, P, P, i64, P, i64, P]
    h.cpe_linear8_create.argtypes = [ctypes.POINTER(P), i32, i32, i32, i32, i32]
    h.cpe_linear8_forward.argtypes = [P, P, i32, P, i64, P, P, i64, P, P, P, i64, P, i64, P, i64]
    h.cpe_linear_create.argtypes = [ctypes.POINTER(P), i32, i32, i32, i32, i32]
    h.cpe_linear_backward8.argtypes = [P, P, i32, P, i64, P, P, i64, P, i64, P, i64, P, P, i64, P, i64, P]
    for name in ("cpe_rms_destroy", "cpe_linear8_destroy", "cpe_linear_destroy"):
        getattr(h, name).argtypes = [P]
    return h


def handle(create, *sizes):
    h = ctypes.c_void_p()
    assert create(ctypes.byref(h), *sizes) == 0
    return h


def check(lib, call, h, good, outputs, allowed=()):
    """Every output in the place of every other argument (pointers are the
    arguments of 4096 and more) but the allowed pairs."""
    pointers = [k for k, v in good.items() if v is not None and v >= 4096]
    before = lib.launches()
    assert call(h, None, *good.values()) == 0 and lib.launches() > before
    for out in outputs:
        for other in pointers:
            if other == out:
                continue
            before = lib.launches()
            got = call(h, None, *{**good, out: good[other]}.values())
            if (out, other) in allowed:
                assert got == 0 and lib.launches() > before, (out, other)
            else:
                assert got == BAD and lib.launches() == before, (out, other)


def test_rms_forward(lib):
    h = handle(lib.cpe_rms_create, 4, 8, 1, 1e-6)
    good = dict(rows=4, x=4096, x_ld=8, residual=8192, residual_ld=8, gamma=12288, sum=16384, sum_ld=8, y=20480, y_ld=8,
                q=24576, q_ld=8, scale=28672, rstd=32768)
    check(lib, lib.cpe_rms_forward, h, good, ("sum", "y", "q", "scale", "rstd"),
          [(o, i) for o in ("sum", "y") for i in ("x", "residual")])
    lib.cpe_rms_destroy(h)


@pytest.mark.parametrize("packed", [False, True])
def test_rms_backward(lib, packed):
    h = handle(lib.cpe_rms_create, 4, 8, 1, 1e-6)
    good = dict(rows=4, h=4096, h_ld=8, h_scale=8192 if packed else None, dy=12288, dy_ld=8, gamma=16384, rstd=20480,
                dsum=24576, dsum_ld=8, dx=28672, dx_ld=8, dgamma=32768)
    check(lib, lib.cpe_rms_backward, h, good, ("dx", "dgamma"),
          [("dx", "dy"), ("dx", "dsum")] + [("dx", "h")] * (not packed))
    lib.cpe_rms_destroy(h)


def test_linear8_forward(lib):
    h = handle(lib.cpe_linear8_create, 4, 8, 8, 1, 2)
    good = dict(rows=4, q=4096, q_ld=8, scale=8192, w=12288, w_ld=8, w_scale=16384, bias=20480, residual=24576,
                residual_ld=8, y=28672, y_ld=8, preact=32768, preact_ld=8)
    check(lib, lib.cpe_linear8_forward, h, good, ("y", "preact"), [("y", "residual")])
    lib.cpe_linear8_destroy(h)


@pytest.mark.parametrize("rows", [4, 4000])
def test_linear_backward8(lib, rows):
    h = handle(lib.cpe_linear_create, rows, 8, 8, 1, 2)
    good = dict(rows=rows, q=1 << 20, q_ld=8, scale=2 << 20, w=3 << 20, w_ld=8, dy=4 << 20, dy_ld=8, zq=5 << 20, zq_ld=8,
                z_scale=6 << 20, dx=7 << 20, dx_ld=8, dw=8 << 20, dw_ld=8, dbias=9 << 20)
    check(lib, lib.cpe_linear_backward8, h, {**good}, ("dx", "dw", "dbias"))
    lib.cpe_linear_destroy(h)
