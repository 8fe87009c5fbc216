"""GPU tests of the integer matrix product (cpe_linear8_*) and of the gradient
from rows in 8 bits (cpe_linear_backward8), against their definitions.

Bounds.  e = 2^-24, u the type's half unit.  The integer sum is exact; z is off
by 3 e |acc s t| for its conversion and the two scales and e |z| for the bias,
an activation passes that on with a slope of at most 1.13 and adds 16 e (|z| + 1),
the output's rounding adds u |y|.

Gradient: dz = dy act'(z) is off by 16 e |dy| (1 + |z|) (z by a rounding, which
that covers).  One operand is rounded to the type: dz (u |dz|, its factor f >= 1
making a subnormal's rounding no larger) with SiLU and GELU in 16 bits, and x
(u |x|) otherwise; in 32 bits x alone, by e.  A sum of n products is off by
(n + 2) e sum|..| in any order, dx by 3 e |dx| more for the factor's division."""
import pytest

from tests.headref import ACTS, DTYPES, E32, TINY, U, activation, activation_grad, inside
from tests.rows8ref import byte_rows, matrix, padded, target, untouched, values

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

#        rows, in, out, pad, lead
SHAPES = [
    (1, 1, 1, 0, 0), (1, 64, 16, 0, 0), (1, 1000, 33, 0, 0), (3, 7, 5, 1, 1), (16, 100, 65, 0, 0), (17, 256, 64, 16, 0),
    (64, 72, 40, 0, 3), (65, 64, 128, 0, 0), (128, 128, 128, 0, 0), (129, 100, 65, 3, 0), (200, 16, 4, 0, 0),
    (300, 257, 131, 0, 0), (257, 520, 136, 24, 0), (1000, 64, 200, 0, 0), (100, 4096, 96, 0, 0), (90, 2049, 130, 0, 0),
    (5000, 24, 8, 0, 0), (12345, 48, 40, 0, 0), (4100, 256, 128, 0, 0), (4097, 512, 64, 16, 0), (6001, 200, 120, 0, 0),
    (9000, 136, 16, 5, 0), (5000, 304, 40, 0, 0), (2, 520, 1032, 0, 0), (33, 130, 70, 5, 0), (64, 1000, 264, 0, 0),
    (48, 96, 2500, 0, 0), (2050, 2064, 2056, 0, 0), (4100, 144, 4104, 16, 0), (700, 16384, 300, 0, 0),
    (3900, 208, 3850, 16, 0), (8100, 16, 1900, 0, 0), (7900, 400, 2001, 0, 0), (300, 1024, 60, 0, 0), (7000, 600, 24, 1, 0),
]


def rows8():
    from paper_2609_16874_amd import rows8 as r
    return r


def head():
    from paper_2609_16874_amd import head as h
    return h


def whole_product(q, w):
    """q w^T as whole numbers (products in 64 bits are exact)."""
    return q.double() @ w.double().t()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_forward(i, dtype):
    M, K, N, pad, lead = SHAPES[i]
    q, s = byte_rows(M, K, i, whole_range=i % 2 == 1)
    w, t = byte_rows(N, K, 100 + i, K ** -0.5)
    if i % 2 == 1:
        s = s / 64
    bias, res = matrix(1, N, "f32", 200 + i)[0], matrix(M, N, dtype, 300 + i)
    dot = whole_product(q, w) * s.double()[:, None] * t.double()
    for act in ACTS:
        for extra in (False, True):
            print(f"linear8 forward {SHAPES[i]} {dtype} {act} {extra}", flush=True)
            h = rows8().Linear8(M + 1, K, N, dtype, act)
            (fy, y), (fz, z) = target(M, N, pad, dtype, lead), target(M, N, pad, dtype, lead)
            assert h.forward(padded(q, pad, lead), s.cuda(), padded(w, pad, lead), t.cuda(),
                             bias.cuda() if extra else None, y, padded(res, pad, lead) if extra else None,
                             z if extra else None) == 0
            want_z = dot + bias.double() if extra else dot
            e_z = 4 * E32 * (dot.abs() + want_z.abs())
            want = activation(act, want_z)
            e_y = 1.13 * e_z + 16 * E32 * (want_z.abs() + 1.0) * (act != "none")
            if extra:
                want = want + res.double()
                inside(z, want_z, e_z + U[dtype] * (want_z.abs() + e_z) + TINY[dtype], "z")
                assert untouched(fz, z)
                e_y = e_y + E32 * (want.abs() + 1.0)
            inside(y, want, e_y + U[dtype] * (want.abs() + e_y) + TINY[dtype], "y")
            assert untouched(fy, y), "written beyond the rows"
            h.close()


@pytest.mark.parametrize("M", [1, 40, 300])
def test_sums_up_to_the_largest(M):
    """65536 products of -128 by -128 (2^30), of -128 by 127, and a lone
    odd one: whole numbers beyond 24 bits, split or not, are exact before
    their rounding."""
    K, N = 65536, 130
    q, w = torch.full((M, K), -128, dtype=torch.int8), torch.full((N, K), -128, dtype=torch.int8)
    w[1], w[2, 5] = 127, -127
    h = rows8().Linear8(M, K, N, "f32")
    y = h.run(q.cuda(), torch.ones(M, device="cuda"), w.cuda(), torch.ones(N, device="cuda")).cpu()
    assert bool((y[:, 3:] == 2.0 ** 30).all()) and bool((y[:, 0] == 2.0 ** 30).all())
    assert bool((y[:, 1] == -(2.0 ** 23) * 127).all()) and bool((y[:, 2] == float(2 ** 30 - 128)).all())
    h.close()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_backward(i, dtype):
    M, K, N, pad, lead = SHAPES[i]
    q, s = byte_rows(M, K, i)
    zq, zs = byte_rows(M, N, 700 + i)
    zq[zq == 0] = 1
    w, dy = matrix(N, K, dtype, 500 + i, K ** -0.5), matrix(M, N, dtype, 600 + i, 0.5)
    x, z = values(q, s), values(zq, zs)
    for act in ACTS:
        print(f"linear backward8 {SHAPES[i]} {dtype} {act}", flush=True)
        h = head().Linear(M, K, N, dtype, act)
        (fx, dx), (fw, dw) = target(M, K, pad, dtype, lead), target(N, K, pad, dtype, lead)
        db = torch.full((N + 1,), 77.0, device="cuda")
        none = act == "none"
        assert h.backward8(padded(q, pad, lead), s.cuda(), padded(w, pad, lead), padded(dy, pad, lead),
                           None if none else padded(zq, pad, lead), None if none else zs.cuda(), dx, dw, db[:N]) == 0
        dz = dy.double() * activation_grad(act, z)
        smooth = act not in ("none", "relu")
        e_f = (16 * E32 * dy.double().abs() * (1.0 + z.abs())) * smooth
        rounds_dz = smooth and dtype != "f32"
        e_dz = e_f + (U[dtype] * dz.abs() * 1.001 + TINY[dtype] + 2 * E32 * dz.abs() if rounds_dz else 0.0)
        e_x = 0.0 if rounds_dz else U[dtype] * x.abs() * 1.001 + TINY[dtype]
        want, mag = dz @ w.double(), dz.abs() @ w.double().abs()
        bound = (N + 2) * E32 * mag + e_dz @ w.double().abs() + 3 * E32 * want.abs() if smooth else (N + 2) * E32 * mag
        inside(dx, want, bound + U[dtype] * (want.abs() + bound) + TINY[dtype], "dx")
        want, mag = dz.t() @ x, dz.abs().t() @ x.abs()
        bound = (M + 2) * E32 * mag
        if smooth:
            bound = bound + e_dz.t() @ x.abs()
        if not rounds_dz:
            bound = bound + (dz.abs() + (e_dz if smooth else 0.0)).t() @ e_x
        inside(dw, want, bound + U[dtype] * (want.abs() + bound) + TINY[dtype], "dw")
        inside(db[:N], dz.sum(0), (M + 2) * E32 * dz.abs().sum(0) + (e_f.sum(0) if smooth else 0.0), "dbias")
        assert untouched(fx, dx) and untouched(fw, dw) and float(db[N]) == 77.0, "written beyond the rows"
        h.close()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu"])
def test_backward_equals_the_one_of_the_unpacked_rows(act, dtype):
    """Where x is the rounded operand it is what unpacking gives."""
    for M, K, N in ((40, 72, 48), (3000, 64, 48), (3000, 264, 200)):
        q, s = (t.cuda() for t in byte_rows(M, K, 1))
        zq, zs = (t.cuda() for t in byte_rows(M, N, 2))
        w, dy = matrix(N, K, dtype, 3).cuda(), matrix(M, N, dtype, 4).cuda()
        h = head().Linear(M, K, N, dtype, act)
        got = h.run_backward8(q, s, w, dy, *((zq, zs) if act == "relu" else ()))
        x = rows8().unpacked(q, s, dtype)
        want = h.run_backward(x, w, dy, rows8().unpacked(zq, zs, dtype) if act == "relu" else None)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), (M, K, N)
        h.close()


def test_gradient_against_differences():
    """An f32 layer's loss, differentiated at the values that its checkpoint
    stands for."""
    for act in ACTS:
        M, K, N = 70, 33, 18
        q, s = byte_rows(M, K, 1)
        x = values(q, s)
        w, dy = matrix(N, K, "f32", 2, K ** -0.5), matrix(M, N, "f32", 3)
        zq, zs = byte_rows(M, N, 4)
        zq[zq == 0] = 1
        z = values(zq, zs)
        h = head().Linear(M, K, N, "f32", act)
        dx, dw, db = (t.cpu().double() for t in h.run_backward8(
            q.cuda(), s.cuda(), w.cuda(), dy.cuda(), *(() if act == "none" else (zq.cuda(), zs.cuda()))))
        g = torch.Generator().manual_seed(5)
        step = 1e-5
        for _ in range(4):
            vx, vw, vb = (torch.randn(t, generator=g, dtype=torch.float64) for t in (x.shape, w.shape, (N,)))

            def loss(t):        # z moves as x w^T + bias does
                u = z + t * vb + (x + t * vx) @ (w.double() + t * vw).t() - x @ w.double().t()
                return float((activation(act, u) * dy.double()).sum())

            slope = (loss(step) - loss(-step)) / (2 * step)
            mine = float((dx * vx).sum() + (dw * vw).sum() + (db * vb).sum())
            assert abs(mine - slope) <= 1e-4 * max(1.0, abs(slope)), act
        h.close()


@pytest.mark.parametrize("M,K,N", [(9, 512, 96), (1500, 64, 48), (1500, 1024, 264)])
@pytest.mark.parametrize("act", ["silu", "none"])
def test_scales_that_are_no_numbers(M, K, N, act):
    """Rows of scale NaN (and 0): z and dw get them, dx and dbias do not take
    them from x; a NaN of the other checkpoint reaches its row of dx."""
    q, s = byte_rows(M, K, 1)
    zq, zs = byte_rows(M, N, 2)
    w, dy = matrix(N, K, "bf16", 3, K ** -0.5).cuda(), matrix(M, N, "bf16", 4).cuda()
    zero = s.clone()
    zero[3] = 0.0
    h = head().Linear(M, K, N, "bf16", act)
    kept = (zq.cuda(), zs.cuda()) if act == "silu" else ()
    dx, dw, db = h.run_backward8(q.cuda(), zero.cuda(), w, dy, *kept)
    assert bool(dx.isfinite().all()) and bool(dw.isfinite().all())
    bad, none = s.clone(), q.clone()
    bad[3], none[3] = float("nan"), 0
    dx2, dw2, db2 = h.run_backward8(none.cuda(), bad.cuda(), w, dy, *kept)
    assert torch.equal(dx2, dx) and torch.equal(db2, db) and bool(dw2.isnan().all())
    if act == "silu":
        bad = zs.clone()
        bad[3] = float("nan")
        dx3, dw3, db3 = h.run_backward8(q.cuda(), zero.cuda(), w, dy, zq.cuda(), bad.cuda())
        rest = torch.arange(M) != 3
        assert bool(dx3[3].isnan().all()) and torch.equal(dx3.cpu()[rest], dx.cpu()[rest]) and bool(db3.isnan().all())
    h.close()
    f = rows8().Linear8(M, K, N, "bf16", act)
    wq, ws = rows8().packed(w)
    y = f.run(q.cuda(), s.cuda(), wq, ws)
    bad = s.clone()
    bad[3] = float("nan")
    y2 = f.run(none.cuda(), bad.cuda(), wq, ws)
    rest = torch.arange(M) != 3
    assert bool(y2[3].isnan().all()) and torch.equal(y2.cpu()[rest], y.cpu()[rest])
    f.close()


def test_residual_in_place_and_single_outputs():
    M, K, N = 100, 64, 32
    q, s, w, t = (v.cuda() for v in byte_rows(M, K, 1) + byte_rows(N, K, 2, 0.1))
    res = matrix(M, N, "f16", 3).cuda()
    h = rows8().Linear8(M, K, N, "f16", "gelu")
    y = h.run(q, s, w, t, residual=res)
    over = res.clone()
    assert h.forward(q, s, w, t, None, over, residual=over) == 0 and torch.equal(over, y)
    e = torch.empty((0, N), dtype=torch.float16, device="cuda")
    assert h.forward(q[:0], s[:0], w, t, None, e) == 0
    h.close()
    lin = head().Linear(M, K, N, "f16", "gelu")
    zq, zs = (v.cuda() for v in byte_rows(M, N, 5))
    wd, dy = matrix(N, K, "f16", 6).cuda(), matrix(M, N, "f16", 7).cuda()
    dx, dw, db = lin.run_backward8(q, s, wd, dy, zq, zs)
    for name, want in (("dx", dx), ("dweight", dw), ("dbias", db)):
        one = torch.empty_like(want)
        assert lin.backward8(q, s, wd, dy, zq, zs, **{name: one}) == 0 and torch.equal(one, want)
    assert lin.backward8(q[:0], s[:0], wd, e, zq[:0], zs[:0], q.half()[:0], dw, db) == 0
    assert float(dw.abs().max()) == 0.0 and float(db.abs().max()) == 0.0
    lin.close()


def test_runs_repeat_and_streams_and_graphs():
    for M, K, N in ((1500, 2048, 64), (9, 512, 96), (3000, 128, 64), (2100, 512, 520)):
        f, h = rows8().Linear8(M, K, N, "f16", "silu"), head().Linear(M, K, N, "f16", "silu")
        w, t = (v.cuda() for v in byte_rows(N, K, 1, K ** -0.5))
        wd, bias = rows8().unpacked(w, t, "f16"), torch.rand(N, device="cuda")
        qs = [[v.cuda() for v in byte_rows(M, K, 10 + i)] for i in range(3)]
        dys = [matrix(M, N, "f16", 20 + i).cuda() for i in range(3)]

        def eager(i):
            y, z = f.run(*qs[i], w, t, bias, keep=True)
            kept = rows8().packed(z)
            return (y, z) + kept + h.run_backward8(*qs[i], wd, dys[i], *kept)

        want = [eager(i) for i in range(3)]
        assert all(torch.equal(a, b) for a, b in zip(want[0], eager(0)))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = eager(1)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want[1], got))
        q, s, dy = qs[0][0].clone(), qs[0][1].clone(), dys[0].clone()
        o = [torch.empty_like(v) for v in want[0]]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            assert f.forward(q, s, w, t, bias, o[0], preact=o[1]) == 0
            assert rows8().pack(o[1], o[2], o[3]) == 0
            assert h.backward8(q, s, wd, dy, o[2], o[3], o[4], o[5], o[6]) == 0
        for step in range(6):
            i = step % 3
            for a, b in ((q, qs[i][0]), (s, qs[i][1]), (dy, dys[i])):
                a.copy_(b)
            for v in o:
                v.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want[i], o)), (step, M)
            if step % 2:
                assert all(torch.equal(a, b) for a, b in zip(want[2 - i], eager(2 - i)))
        f.close()
        h.close()


@pytest.mark.parametrize("N", [16, 136, 264])
def test_offsets_beyond_32_bits(N):
    """4,500,000 rows of 1024 bytes: 4.6e9 of them; equal rows far apart give
    equal outputs."""
    M, K = 4_500_000, 1024
    n = M // 10
    part = torch.randint(-127, 128, (n, K), dtype=torch.int8, device="cuda")
    q, s = part.repeat(10, 1), torch.full((M,), 0.02, device="cuda")
    w, t = (v.cuda() for v in byte_rows(N, K, 2, K ** -0.5))
    h = rows8().Linear8(M, K, N, "bf16")
    y = h.run(q, s, w, t)
    want = values(part[:1000], s[:1000]) @ values(w, t).t()
    assert float((y[:1000].double() - want).abs().max()) <= 2.0 ** -8 * float(want.abs().max())
    assert torch.equal(y[-n:], y[:n])
    h.close()
    lin = head().Linear(M, K, N, "bf16")
    dx, dw, _ = lin.run_backward8(q, s, rows8().unpacked(w, t, "bf16"), y)
    assert torch.equal(dx[-n:], dx[:n])
    lin.close()
