"""GPU tests of the RMS norm (cpe_rms_*) against its definition in 64 bits.

Bounds.  e = 2^-24, u the type's half unit.  A thread adds at most 16 squares
(64 / 4 vectors of 4, or 16 of two vectors of 8), and at most 6 steps within
its wave and 16 waves follow: the sum of squares, all of one sign, is off by at
most 40 e, half of that in the root, and 6 e more for the mean, eps, the root,
its reciprocal and the two products: y is off by 26 e, rstd by 25 e.  The sum
with the residual is one binary32 addition, rounded: exact.

Gradient, with t = dy gamma and xh = h rstd (rstd an input): xh is off by 2 e
(3 with a scale), t by e, a = sum t xh / C by 44 e sum|t xh| / C, so dx by
  rstd (4 e |t| + |xh| (44 e A + 8 e |a|)) + 2 e |dsum|,  A = sum |t xh| / C,
and the output's rounding; dgamma by (rows + 8) e sum |dy xh|."""
import pytest

from tests.headref import DTYPES, E32, TINY, U, inside
from tests.rows8ref import byte_rows, check_packed, matrix, padded, target, untouched, values

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

EPS = 1e-6
#        rows, channels, pad, lead
SHAPES = [
    (1, 1, 0, 0), (1, 1024, 0, 0), (3, 5, 2, 1), (5, 8, 0, 0), (70, 9, 0, 0), (40, 63, 1, 2), (333, 64, 0, 0), (300, 65, 3, 1),
    (17, 100, 0, 0), (1000, 127, 0, 0), (129, 256, 8, 0), (64, 511, 0, 0), (3000, 512, 0, 0), (10, 1001, 3, 1),
    (700, 1024, 0, 0), (2, 2049, 0, 0), (65, 4096, 0, 0), (3, 4104, 0, 0), (4, 8191, 0, 1), (5, 10000, 24, 0), (2, 16384, 0, 0),
    (70001, 24, 0, 0), (30000, 260, 4, 0), (12000, 100, 12, 0),
    (1500, 2500, 0, 0), (900, 4100, 8, 0), (700, 7000, 0, 1), (600, 9000, 0, 0),    # (several turns of a workgroup per row)
]


def rows8():
    from paper_2609_16874_amd import rows8 as r
    return r


def norm64(h, gamma):
    rstd = 1.0 / torch.sqrt((h * h).mean(1) + EPS)
    return h * rstd[:, None] * gamma, rstd


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_forward(i, dtype):
    M, C, pad, lead = SHAPES[i]
    x, res = matrix(M, C, dtype, i, 1.5), matrix(M, C, dtype, 100 + i)
    gamma = 1.0 + 0.3 * matrix(1, C, "f32", 200 + i)[0]
    norm = rows8().RmsNorm(M + 1, C, dtype, EPS)
    for extra in (False, True):
        print(f"rms forward {SHAPES[i]} {dtype} {extra}", flush=True)
        fs, total = target(M, C, pad, dtype, lead)
        fy, y = target(M, C, pad, dtype, lead)
        fq, q = target(M, C, pad, "i8", lead)
        scale, rstd = (torch.full((M + 1,), 77.0, device="cuda") for _ in range(2))
        assert norm.forward(padded(x, pad, lead), gamma.cuda() if extra else None,
                            padded(res, pad, lead) if extra else None, total, y, q, scale[:M], rstd[:M]) == 0
        h = (x.float() + res.float()).to(DTYPES[dtype]) if extra else x
        assert torch.equal(total.cpu(), h)
        want, r = norm64(h.double(), gamma.double() if extra else 1.0)
        inside(rstd[:M], r, 25 * E32 * r, "rstd")
        inside(y, want, 26 * E32 * want.abs() + U[dtype] * (1 + 26 * E32) * want.abs() + TINY[dtype], "y")
        check_packed(q, scale[:M], want, 26 * E32)
        assert untouched(fs, total) and untouched(fy, y) and untouched(fq, q)
        assert float(scale[M]) == 77.0 and float(rstd[M]) == 77.0
    norm.close()


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_backward(i, dtype, packed):
    M, C, pad, lead = SHAPES[i]
    q, scale = byte_rows(M, C, i, 1.5)
    x = matrix(M, C, dtype, 50 + i, 1.5)
    dy, dsum = matrix(M, C, dtype, 300 + i, 0.5), matrix(M, C, dtype, 400 + i, 0.5)
    gamma = 1.0 + 0.3 * matrix(1, C, "f32", 200 + i)[0]
    h = values(q, scale) if packed else x.double()
    rstd = (1.0 / torch.sqrt((h * h).mean(1) + EPS)).float()
    norm = rows8().RmsNorm(M + 1, C, dtype, EPS)
    for extra in (False, True):
        print(f"rms backward {SHAPES[i]} {dtype} {packed} {extra}", flush=True)
        fx, dx = target(M, C, pad, dtype, lead)
        dgamma = torch.full((C + 1,), 77.0, device="cuda")
        assert norm.backward(padded(q if packed else x, pad, lead), padded(dy, pad, lead), gamma.cuda() if extra else None,
                             rstd.cuda(), dx, dgamma[:C], padded(dsum, pad, lead) if extra else None,
                             scale.cuda() if packed else None) == 0
        R = rstd.double()[:, None]
        t, xh = dy.double() * (gamma.double() if extra else 1.0), h * R
        a, A = (t * xh).mean(1, keepdim=True), (t * xh).abs().mean(1, keepdim=True)
        want = R * (t - xh * a)
        bound = R * (4 * E32 * t.abs() + xh.abs() * (44 * E32 * A + 8 * E32 * a.abs()))
        if extra:
            want = want + dsum.double()
            bound = bound + 2 * E32 * (dsum.double().abs() + want.abs())
        inside(dx, want, bound + U[dtype] * (want.abs() + bound) + TINY[dtype], "dx")
        inside(dgamma[:C], (dy.double() * xh).sum(0), (M + 8) * E32 * (dy.double() * xh).abs().sum(0), "dgamma")
        assert untouched(fx, dx) and float(dgamma[C]) == 77.0
    norm.close()


def test_gradient_against_differences():
    """x, the residual and gamma moved along random directions; the loss takes
    the output and the sum itself."""
    M, C = 37, 75
    x, res, dy, dsum = (matrix(M, C, "f32", i) for i in range(4))
    gamma = 1.0 + 0.3 * matrix(1, C, "f32", 5)[0]
    norm = rows8().RmsNorm(M, C, "f32", EPS)
    total, y, rstd = norm.run(x.cuda(), gamma.cuda(), res.cuda())
    dx, dgamma = (t.cpu().double() for t in norm.run_backward(total, dy.cuda(), gamma.cuda(), rstd, dsum.cuda()))
    g = torch.Generator().manual_seed(5)
    step = 1e-5
    for _ in range(6):
        vx, vr, vg = (torch.randn(s, generator=g, dtype=torch.float64) for s in (x.shape, x.shape, gamma.shape))

        def loss(t):
            h = x.double() + res.double() + t * (vx + vr)
            return float((norm64(h, gamma.double() + t * vg)[0] * dy.double() + h * dsum.double()).sum())

        slope = (loss(step) - loss(-step)) / (2 * step)
        mine = float((dx * (vx + vr)).sum() + (dgamma * vg).sum())
        assert abs(mine - slope) <= 1e-4 * max(1.0, abs(slope))
    norm.close()


@pytest.mark.parametrize("C", [3, 100, 1024, 3000, 12000])
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_in_place(C, dtype):
    """The sum in the residual's place and y in x's; dx in those of dy, of the
    gradient past the norm and of h."""
    M = 77
    x, res, dy, ds = (matrix(M, C, dtype, i).cuda() for i in range(4))
    gamma = 1.0 + 0.3 * matrix(1, C, "f32", 5)[0].cuda()
    norm = rows8().RmsNorm(M, C, dtype, EPS)
    total, y, rstd = norm.run(x, gamma, res)
    a, b = x.clone(), res.clone()
    assert norm.forward(a, gamma, b, sum=b, y=a) == 0
    assert torch.equal(a, y) and torch.equal(b, total)
    a, b = x.clone(), res.clone()
    assert norm.forward(a, gamma, b, sum=a, y=b) == 0
    assert torch.equal(a, total) and torch.equal(b, y)
    dx, dgamma = norm.run_backward(total, dy, gamma, rstd, ds)
    for which in range(3):
        t = [total.clone(), dy.clone(), ds.clone()]
        dg = torch.empty_like(dgamma)
        assert norm.backward(t[0], t[1], gamma, rstd, t[which], dg, t[2]) == 0
        assert torch.equal(t[which], dx) and torch.equal(dg, dgamma)
    norm.close()


@pytest.mark.parametrize("C", [7, 64, 1000, 5000])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_rows_of_extreme_values(C, dtype):
    """A NaN, an infinity, zeros: they stay in their rows."""
    M = 40
    x = matrix(M, C, dtype, 1)
    norm = rows8().RmsNorm(M, C, dtype, EPS)
    y, rstd = norm.run(x.cuda(), None)
    (q, scale), _ = norm.run(x.cuda(), None, packed=True)
    z = x.clone()
    z[3, C // 2], z[5, C - 1], z[6] = float("nan"), float("inf"), 0.0
    y2, rstd2 = norm.run(z.cuda(), None)
    (q2, scale2), _ = norm.run(z.cuda(), None, packed=True)
    rest = torch.ones(M, dtype=torch.bool)
    rest[3] = rest[5] = rest[6] = False
    assert torch.equal(y2.cpu()[rest], y.cpu()[rest]) and torch.equal(q2.cpu()[rest], q.cpu()[rest])
    assert torch.equal(scale2.cpu()[rest], scale.cpu()[rest]) and torch.equal(rstd2.cpu()[rest], rstd.cpu()[rest])
    assert bool(y2[3].isnan().all()) and float(rstd2[5]) == 0.0
    assert bool(y2[5, C - 1].isnan()) and bool((y2[5, :C - 1] == 0).all())
    assert bool(scale2[3].isnan()) and bool(scale2[5].isnan()) and bool((q2[3:6:2] == 0).all())
    assert bool((y2[6] == 0).all()) and bool((q2[6] == 0).all()) and not bool(scale2[6].isnan())
    # the gradient: a NaN of dy reaches its row and its column of dgamma
    dy = matrix(M, C, dtype, 2)
    dx, dg = norm.run_backward(x.cuda(), dy.cuda(), None, rstd)
    dy[4, C // 2] = float("nan")
    dx2, dg2 = norm.run_backward(x.cuda(), dy.cuda(), None, rstd)
    assert bool(dx2[4].isnan().all()) and bool(dg2[C // 2].isnan()) and int(dg2.isnan().sum()) == 1
    rest = torch.arange(M) != 4
    assert torch.equal(dx2.cpu()[rest], dx.cpu()[rest])
    norm.close()


def test_outputs_by_themselves_and_no_rows():
    M, C = 600, 136
    norm = rows8().RmsNorm(M, C, "bf16", EPS)
    x, res, dy = (matrix(M, C, "bf16", i).cuda() for i in range(3))
    gamma = 1.0 + 0.3 * matrix(1, C, "f32", 5)[0].cuda()
    total, y, rstd = norm.run(x, gamma, res)
    _, (q, scale), _ = norm.run(x, gamma, res, packed=True)
    one = torch.empty_like(y)
    assert norm.forward(x, gamma, res, y=one) == 0 and torch.equal(one, y)
    assert norm.forward(x, gamma, res, sum=one) == 0 and torch.equal(one, total)
    q1, s1 = torch.empty_like(q), torch.empty_like(scale)
    assert norm.forward(x, gamma, res, q=q1, scale=s1) == 0 and torch.equal(q1, q) and torch.equal(s1, scale)
    dx, dg = norm.run_backward(total, dy, gamma, rstd)
    assert norm.backward(total, dy, gamma, rstd, dx=one) == 0 and torch.equal(one, dx)
    only = torch.empty_like(dg)
    assert norm.backward(total, dy, gamma, rstd, dgamma=only) == 0 and torch.equal(only, dg)
    e, r = torch.empty((0, C), dtype=torch.bfloat16, device="cuda"), torch.empty(0, device="cuda")
    assert norm.forward(e, gamma, y=e) == 0
    assert norm.backward(e, e, gamma, r, dx=e, dgamma=only) == 0 and float(only.abs().max()) == 0.0
    assert norm.backward(e, e, gamma, r, dx=e) == 0
    norm.close()


def test_runs_repeat_and_streams_and_graphs():
    for M, C in ((2000, 320), (3, 6000)):
        norm = rows8().RmsNorm(M, C, "f16", EPS)
        gamma = 1.0 + 0.3 * matrix(1, C, "f32", 5)[0].cuda()
        xs, rs, ds = ([matrix(M, C, "f16", s + i).cuda() for i in range(3)] for s in (10, 20, 30))

        def eager(i):
            total, (q, scale), rstd = norm.run(xs[i], gamma, rs[i], packed=True)
            return (total, q, scale, rstd) + norm.run_backward(total, ds[i], gamma, rstd, ds[i])

        want = [eager(i) for i in range(3)]
        assert all(torch.equal(a, b) for a, b in zip(want[0], eager(0)))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = eager(1)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want[1], got))
        x, r, d = xs[0].clone(), rs[0].clone(), ds[0].clone()
        outs = [torch.empty_like(t) for t in want[0]]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            assert norm.forward(x, gamma, r, sum=outs[0], q=outs[1], scale=outs[2], rstd=outs[3]) == 0
            assert norm.backward(outs[0], d, gamma, outs[3], outs[4], outs[5], d) == 0
        for step in range(6):
            i = step % 3
            for t, v in ((x, xs), (r, rs), (d, ds)):
                t.copy_(v[i])
            for t in outs:
                t.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want[i], outs)), step
            if step % 2:
                assert all(torch.equal(a, b) for a, b in zip(want[2 - i], eager(2 - i)))
        norm.close()


def test_offsets_beyond_32_bits():
    """4.4e9 elements: equal rows far apart give equal outputs."""
    n, C = 5000, 4900
    part, gamma = matrix(n, C, "bf16", 4).cuda(), 1.0 + 0.3 * matrix(1, C, "f32", 5)[0].cuda()
    M = 180 * n
    x = part.repeat(180, 1)
    norm = rows8().RmsNorm(M, C, "bf16", EPS)
    y, rstd = norm.run(x, gamma)
    want, r = norm64(part.double(), gamma.double())
    inside(y[-n:], want.cpu(), (26 * E32 + 1.001 * U["bf16"]) * want.cpu().abs(), "y")
    assert torch.equal(y[:n], y[-n:]) and torch.equal(rstd[:n], rstd[-n:])
    dx, dgamma = norm.run_backward(x, y, gamma, rstd)
    assert torch.equal(dx[:n], dx[-n:])
    xh = part.double() * r[:, None]
    want = 180 * (want.to(torch.bfloat16).double() * xh).sum(0)
    assert float(((dgamma.double() - want) / want).abs().max()) <= 2.0 ** -8
    norm.close()


@pytest.mark.parametrize("C", [64, 512, 4096])
def test_rows_that_the_caches_do_not_hold(C):
    """150 M elements, written past the caches: the same rows in pieces, which
    are not, give the same bits; dgamma to the sums' bound."""
    M = (150 << 20) // C
    g = torch.Generator(device="cuda").manual_seed(1)
    x, res, dy = (torch.randn((M, C), generator=g, device="cuda").half() for _ in range(3))
    gamma = 1.0 + 0.3 * matrix(1, C, "f32", 5)[0].cuda()
    norm = rows8().RmsNorm(M, C, "f16", EPS)
    total, y, rstd = norm.run(x, gamma, res)
    _, (q, scale), _ = norm.run(x, gamma, res, packed=True)
    kept, kept_scale = rows8().packed(total)
    dx, dgamma = norm.run_backward(total, dy, gamma, rstd, res)
    dx8, _ = norm.run_backward(kept, dy, gamma, rstd, res, kept_scale)
    sums, most, each = 0.0, 0.0, -(-M // 5)
    for lo in range(0, M, each):
        p = slice(lo, min(M, lo + each))
        t, u, r = norm.run(x[p], gamma, res[p])
        _, (b, s), _ = norm.run(x[p], gamma, res[p], packed=True)
        assert torch.equal(t, total[p]) and torch.equal(u, y[p]) and torch.equal(r, rstd[p])
        assert torch.equal(b, q[p]) and torch.equal(s, scale[p])
        d, dg = norm.run_backward(t, dy[p], gamma, r, res[p])
        assert torch.equal(d, dx[p])
        assert torch.equal(norm.run_backward(kept[p], dy[p], gamma, r, res[p], kept_scale[p])[0], dx8[p])
        sums = sums + dg.double()
        most = most + (dy[p].double() * t.double() * r.double()[:, None]).abs().sum(0)
    assert bool(((dgamma.double() - sums).abs() <= 2 * (M + 8) * E32 * most).all())
    norm.close()
