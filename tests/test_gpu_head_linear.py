"""GPU tests of the matrix product (cpe_linear_*) against its definition in 64
bits.

Bounds.  e = 2^-24, u the type's half unit.  A sum of K products in any order
is off by at most (K + 2) e sum|x w| (K e at worst, the products of 16-bit
factors being exact; 2 e for the bias and rounding); an activation passes an
error on with a slope of at most 1.13 and adds 16 e (|z| + 1); the output's
rounding adds u |y|.  In the gradient dz = dy act'(z) is off by
16 e |dy| (1 + |z|), and as an operand by another u |dz|."""
import pytest

from tests.headref import ACTS, DTYPES, E32, TINY, U, activation, activation_grad, inside

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

#        rows, in, out, pad
SHAPES = [
    (1, 1, 1, 0), (1, 64, 16, 0), (1, 1000, 33, 0), (3, 7, 5, 1), (16, 100, 65, 0), (17, 256, 64, 8),
    (64, 72, 40, 0), (65, 64, 128, 0), (128, 128, 128, 0), (129, 100, 65, 3), (200, 8, 4, 0), (300, 257, 131, 0),
    (257, 520, 136, 24), (1000, 64, 200, 0), (100, 4096, 96, 0), (90, 2049, 130, 0), (5000, 24, 8, 0),
    (12345, 48, 40, 0), (4100, 256, 128, 0), (4097, 512, 64, 8), (6001, 200, 120, 0), (9000, 136, 16, 5), (5000, 304, 40, 0),
    (2, 520, 1032, 0), (33, 130, 70, 5), (64, 1000, 264, 0), (48, 96, 2500, 0),
    (2050, 2072, 2056, 0), (4100, 136, 4104, 8),
]


def head():
    from paper_2609_16874_amd import head as h
    return h


def matrix(rows, width, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn((rows, width), generator=g)).to(DTYPES[dtype])


def padded(m, pad):
    full = torch.full((m.shape[0], m.shape[1] + pad), float("nan"), dtype=m.dtype, device="cuda")
    full[:, :m.shape[1]] = m.cuda()
    return full[:, :m.shape[1]]


def target(rows, width, pad, dtype):
    return torch.full((rows, width + pad), 77.0, dtype=DTYPES[dtype], device="cuda")


def whole(full, width):
    return bool((full[:, width:] == 77.0).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_forward(i, dtype):
    M, K, N, pad = SHAPES[i]
    x, w = matrix(M, K, dtype, i), matrix(N, K, dtype, 100 + i, K ** -0.5)
    bias, res = matrix(1, N, "f32", 200 + i)[0], matrix(M, N, dtype, 300 + i)
    dot, mag = x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t()
    for act in ACTS:
        for extra in (False, True):
            print(f"linear forward {SHAPES[i]} {dtype} {act} {extra}", flush=True)
            h = head().Linear(M + 1, K, N, dtype, act)
            y, z = target(M, N, pad, dtype), target(M, N, pad, dtype)
            st = h.forward(padded(x, pad), padded(w, pad), bias.cuda() if extra else None, y[:, :N],
                           padded(res, pad) if extra else None, z[:, :N] if extra else None)
            assert st == 0
            want_z = dot + bias.double() if extra else dot
            e_z = (K + 2) * E32 * (mag + bias.double().abs())
            want = activation(act, want_z)
            e_y = 1.13 * e_z + 16 * E32 * (want_z.abs() + 1.0) * (act != "none")
            if extra:
                want = want + res.double()
                inside(z[:, :N], want_z, e_z + U[dtype] * (want_z.abs() + e_z) + TINY[dtype], "z")
                assert whole(z, N)
                e_y = e_y + E32 * (want.abs() + 1.0)
            inside(y[:, :N], want, e_y + U[dtype] * (want.abs() + e_y) + TINY[dtype], "y")
            assert whole(y, N), "written beyond the rows"
            h.close()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_backward(i, dtype):
    M, K, N, pad = SHAPES[i]
    x, w = matrix(M, K, dtype, 400 + i), matrix(N, K, dtype, 500 + i, K ** -0.5)
    dy, z = matrix(M, N, dtype, 600 + i, 0.5), matrix(M, N, dtype, 700 + i)
    z[z == 0] = 1.0
    for act in ACTS:
        print(f"linear backward {SHAPES[i]} {dtype} {act}", flush=True)
        h = head().Linear(M, K, N, dtype, act)
        dx, dw = target(M, K, pad, dtype), target(N, K, pad, dtype)
        db = torch.full((N,), 77.0, device="cuda")
        assert h.backward(padded(x, pad), padded(w, pad), padded(dy, pad),
                          None if act == "none" else padded(z, pad), dx[:, :K], dw[:, :K], db) == 0
        dz = dy.double() * activation_grad(act, z.double())
        e_f = (16 * E32 * dy.double().abs() * (1.0 + z.double().abs())) * (act not in ("none", "relu"))
        e_dz = e_f + (U[dtype] * dz.abs() + TINY[dtype] if act not in ("none", "relu") and dtype != "f32" else 0.0)
        want, mag = dz @ w.double(), dz.abs() @ w.double().abs()
        bound = (N + 2) * E32 * mag + e_dz @ w.double().abs()
        inside(dx[:, :K], want, bound + U[dtype] * (want.abs() + bound) + TINY[dtype], "dx")
        want, mag = dz.t() @ x.double(), dz.abs().t() @ x.double().abs()
        bound = (M + 2) * E32 * mag + e_dz.t() @ x.double().abs()
        inside(dw[:, :K], want, bound + U[dtype] * (want.abs() + bound) + TINY[dtype], "dw")
        inside(db, dz.sum(0), (M + 2) * E32 * dz.abs().sum(0) + e_f.sum(0), "dbias")
        assert whole(dx, K) and whole(dw, K), "written beyond the rows"
        h.close()


@pytest.mark.parametrize("act", ACTS)
def test_gradient_against_differences(act):
    M, K, N = 70, 33, 18
    x, w, dy = matrix(M, K, "f32", 1), matrix(N, K, "f32", 2, K ** -0.5), matrix(M, N, "f32", 3)
    bias = matrix(1, N, "f32", 4)[0]
    h = head().Linear(M, K, N, "f32", act)
    _, z = h.run(x.cuda(), w.cuda(), bias.cuda(), keep=True)
    dx, dw, db = (t.cpu().double() for t in h.run_backward(x.cuda(), w.cuda(), dy.cuda(), z))
    g = torch.Generator().manual_seed(5)
    step = 1e-5
    for _ in range(6):
        vx, vw, vb = (torch.randn(s, generator=g, dtype=torch.float64) for s in (x.shape, w.shape, bias.shape))

        def loss(t):
            u = (x.double() + t * vx) @ (w.double() + t * vw).t() + bias.double() + t * vb
            return float((activation(act, u) * dy.double()).sum())

        slope = (loss(step) - loss(-step)) / (2 * step)
        mine = float((dx * vx).sum() + (dw * vw).sum() + (db * vb).sum())
        assert abs(mine - slope) <= 1e-4 * max(1.0, abs(slope)) + (0.05 if act == "relu" else 0.0)
    h.close()


def test_no_rows_and_single_outputs():
    h = head().Linear(64, 40, 24, "bf16", "silu")
    x, w = torch.empty((0, 40), dtype=torch.bfloat16, device="cuda"), matrix(24, 40, "bf16", 1).cuda()
    e = torch.empty((0, 24), dtype=torch.bfloat16, device="cuda")
    assert h.forward(x, w, None, e) == 0
    dw, db = torch.full_like(w, 7.0), torch.full((24,), 7.0, device="cuda")
    assert h.backward(x, w, e, e, torch.empty_like(x), dw, db) == 0
    assert float(dw.abs().max()) == 0.0 and float(db.abs().max()) == 0.0
    x, dy, z = (matrix(50, s, "bf16", 2 + s).cuda() for s in (40, 24, 24))
    dx, dw, db = h.run_backward(x, w, dy, z)
    one = torch.empty_like(dx)
    assert h.backward(x, w, dy, z, dx=one) == 0 and torch.equal(one, dx)
    one = torch.empty_like(dw)
    assert h.backward(x, w, dy, z, dweight=one) == 0 and torch.equal(one, dw)
    one = torch.empty_like(db)
    assert h.backward(x, w, dy, z, dbias=one) == 0 and torch.equal(one, db)
    h.close()


@pytest.mark.parametrize("N", [24, 136])
def test_pointers_off_16_bytes(N):
    """Rows that start one element into their buffers."""
    M, K = 300, 72
    h = head().Linear(M, K, N, "f16", "relu")
    x, w, dy, z = (matrix(a, b, "f16", 40 + i) for i, (a, b) in enumerate(((M, K), (N, K), (M, N), (M, N))))

    def off(m):
        full = torch.full((m.shape[0], m.shape[1] + 1), float("nan"), dtype=m.dtype, device="cuda")
        full[:, 1:] = m.cuda()
        return full[:, 1:]

    y = h.run(x.cuda(), w.cuda())
    other = torch.full((M, N + 1), 77.0, dtype=torch.float16, device="cuda")
    assert h.forward(off(x), off(w), None, other[:, 1:]) == 0
    # (the two may add up in other orders: a unit of the sums' rounding apart)
    assert float((other[:, 1:].float() - y.float()).abs().max()) <= 2.0 ** -10 * float(y.abs().max())
    assert bool((other[:, 0] == 77.0).all())
    for a, b in zip(h.run_backward(x.cuda(), w.cuda(), dy.cuda(), z.cuda()),
                    h.run_backward(off(x), off(w), off(dy), off(z))):
        assert float((a.float() - b.float()).abs().max()) <= 2.0 ** -10 * float(a.abs().max())
    h.close()


def test_residual_in_place_and_infinities():
    x, w, res = matrix(100, 64, "f16", 1), matrix(32, 64, "f16", 2, 0.125), matrix(100, 32, "f16", 3)
    h = head().Linear(100, 64, 32, "f16", "gelu")
    y = h.run(x.cuda(), w.cuda(), residual=res.cuda())
    over = res.cuda().clone()
    assert h.forward(x.cuda(), w.cuda(), None, over, residual=over) == 0
    assert torch.equal(over, y)
    x[5, 6] = float("nan")
    x[7, 8] = float("inf")
    y2 = h.run(x.cuda(), w.cuda(), residual=res.cuda())
    rest = torch.ones(100, dtype=torch.bool)
    rest[5] = rest[7] = False
    assert bool(y2[5].isnan().all()) and not bool(y2[7].isfinite().all())
    assert torch.equal(y2.cpu()[rest], y.cpu()[rest])
    h.close()


def test_runs_repeat_and_streams_and_graphs():
    """Two runs agree bit for bit; a side stream and every replay of a graph
    give the eager result, with eager calls in between; split and whole
    products, the few-row form and the bias gradient."""
    for M, K, N in ((1500, 1024, 64), (9, 512, 96)):
        h = head().Linear(M, K, N, "f16", "silu")
        w, bias = matrix(N, K, "f16", 1, K ** -0.5).cuda(), torch.rand(N, device="cuda")
        xs = [matrix(M, K, "f16", 10 + i).cuda() for i in range(3)]
        dys = [matrix(M, N, "f16", 20 + i).cuda() for i in range(3)]

        def eager(i):
            y, z = h.run(xs[i], w, bias, keep=True)
            return (y, z) + h.run_backward(xs[i], w, dys[i], z)

        want = [eager(i) for i in range(3)]
        assert all(torch.equal(a, b) for a, b in zip(want[0], eager(0)))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = eager(1)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want[1], got))
        x, dy = xs[0].clone(), dys[0].clone()
        outs = [torch.empty_like(t) for t in want[0]]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            assert h.forward(x, w, bias, outs[0], preact=outs[1]) == 0
            assert h.backward(x, w, dy, outs[1], outs[2], outs[3], outs[4]) == 0
        for step in range(6):
            i = step % 3
            x.copy_(xs[i])
            dy.copy_(dys[i])
            for t in outs:
                t.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want[i], outs)), step
            if step % 2:
                assert all(torch.equal(a, b) for a, b in zip(want[2 - i], eager(2 - i)))
        h.close()


@pytest.mark.parametrize("N", [16, 136])
def test_offsets_beyond_32_bits(N):
    """2,200,000 rows of 1024 features: 2.25e9 elements; equal rows far apart
    give equal outputs (narrow and tiled products)."""
    M, K = 2_200_000, 1024
    n = M // 10
    g = torch.Generator(device="cuda").manual_seed(1)
    part = torch.randn((n, K), generator=g, device="cuda").to(torch.bfloat16)
    x = part.repeat(10, 1)
    w = matrix(N, K, "bf16", 2, K ** -0.5).cuda()
    h = head().Linear(M, K, N, "bf16")
    y = h.run(x, w)
    want = part[:1000].float() @ w.float().t()
    assert float((y[:1000].float() - want).abs().max()) <= 2.0 ** -8 * float(want.abs().max()) + 1e-4
    assert torch.equal(y[-n:], y[:n])
    dx, dw, _ = h.run_backward(x, w, y)
    assert torch.equal(dx[-n:], dx[:n])
    h.close()
