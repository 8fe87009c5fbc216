"""GPU tests of the group norm (cpe_norm_*) against its definition in 64 bits.

Bounds.  With e = 2^-24, u the output type's half unit: a statistic is summed
over chains of at most 128 additions and merged, so the mean is off by less
than 128 e max|x - mean| + 2 e |mean| and rstd, whose relative error is half
the variance's, by 256 e; those pass into xh = (x - mean) rstd with another
6 e |xh|, into u and y through slopes of at most |gamma| and 1.13 (the largest
slope of GELU; SiLU's is 1.10), plus 16 e (|u| + 1) for the activation itself.
The gradient's terms follow the same chain with second derivatives below 1."""
import math
import random

import pytest

from tests.headref import ACTS, DTYPES, E32, TINY, U, inside, norm, norm_grad, norm_sample

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
EPS = 1e-5

#        B, P, C, G, pad, sizes
SHAPES = [
    (1, 1, 1, 1, 0, None),                     # one value: xh is 0
    (1, 1, 64, 8, 0, None),                    # one pixel
    (2, 3, 10, 5, 0, None),
    (1, 257, 64, 8, 0, None),
    (1, 1000, 7, 7, 0, None),                  # vectors of one channel, groups of one
    (3, 100, 100, 25, 3, None),                # rows that no vector boundary fits
    (2, 33, 1024, 32, 8, None),
    (1, 9, 8192, 1, 0, None),                  # the widest row, one group
    (1, 5, 4100, 41, 0, None),                 # several column steps, the last partial
    (4, 64, 96, 12, 0, (0, 1, 64, 70)),        # an empty sample, one pixel, all, a count beyond the map
    (3, 40, 24, 2, 1, (-3, 17, 39)),
    (1, 70001, 16, 2, 0, None),
    (70, 11, 32, 4, 0, None),
    (90, 11, 32, 8, 0, None),                  # more groups than workgroups at once
    (2, 20011, 125, 25, 0, None),              # 16-byte vectors that end across the row's end
    (1, 30001, 13, 13, 2, (29000,)),
    (1, 9001, 2053, 1, 0, None),
    (40, 1201, 36, 9, 0, None),                # many samples of several workgroups each
]


def head():
    from paper_2609_16874_amd import head as h
    return h


def make(B, P, C, pad, dtype, seed, scale=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    v = scale * torch.randn((B, P, C + pad), generator=g) + shift
    return v.to(DTYPES[dtype])


def bounds_y(x, gamma, beta, G, act, sizes, dtype, want):
    B, P, C = x.shape
    out = torch.zeros_like(x)
    for b, n in enumerate(sizes):
        if n == 0:
            continue
        _, mean, rstd = norm_sample(x[b, :n], gamma, beta, G, act, EPS)
        m, r = mean.repeat_interleave(C // G), rstd.repeat_interleave(C // G)
        spread = (x[b, :n] - m).abs().amax(0).reshape(G, -1).amax(1).repeat_interleave(C // G)
        xh = ((x[b, :n] - m) * r).abs()
        e_xh = r * (128 * E32 * spread + 2 * E32 * m.abs()) + (256 + 6) * E32 * xh
        u = xh * gamma.abs() + beta.abs()
        out[b, :n] = 1.13 * (gamma.abs() * e_xh + 2 * E32 * u) + 16 * E32 * (u + 1.0)
    return out + U[dtype] * (want.abs() + out) + TINY[dtype]


def inputs(shape, dtype, seed=0, scale=1.0, shift=0.0):
    B, P, C, G, pad, sizes = shape
    x = make(B, P, C, pad, dtype, seed, scale, shift)[..., :C]
    g = torch.Generator().manual_seed(seed + 1)
    gamma, beta = 1.0 + 0.3 * torch.randn(C, generator=g), 0.3 * torch.randn(C, generator=g)
    real = [P] * B if sizes is None else [min(max(s, 0), P) for s in sizes]
    valid = None if sizes is None else torch.tensor(sizes, dtype=torch.int32, device="cuda")
    return x, gamma, beta, valid, real


def behind(x, sizes, value):
    """A copy with `value` in the places behind each sample's pixels."""
    x = x.clone()
    for b, n in enumerate(sizes):
        x[b, n:] = value
    return x


def padded(x, pad, fill=float("nan")):
    """The map on the GPU, its rows inside a wider buffer."""
    full = torch.full(x.shape[:-1] + (x.shape[-1] + pad,), fill, dtype=x.dtype, device="cuda")
    full[..., :x.shape[-1]] = x.cuda()
    return full[..., :x.shape[-1]]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_forward(i, dtype):
    shape = SHAPES[i]
    B, P, C, G, pad, sizes = shape
    for act in ACTS:
        print(f"norm forward {shape} {dtype} {act}", flush=True)
        x, gamma, beta, valid, real = inputs(shape, dtype, seed=i)
        xg = padded(behind(x, real, float("nan")), pad)
        y = torch.full((B, P, C + pad), 77.0, dtype=x.dtype, device="cuda")
        h = head().GroupNorm(B, P, C, G, dtype, act, EPS)
        stats = torch.full((B, G, 2), 77.0, device="cuda")
        assert h.forward(xg, gamma.cuda(), beta.cuda(), y[..., :C], stats, valid) == 0
        x64 = behind(x, real, 0.0).double()
        want, st = norm(x64, gamma.double(), beta.double(), G, act, EPS, real)
        inside(y[..., :C], want, bounds_y(x64, gamma.double(), beta.double(), G, act, real, dtype, want), "y")
        assert bool((y[..., C:] == 77.0).all()), "written beyond the rows"
        spread = x64.abs().max() + 1.0
        inside(stats[..., 0], st[..., 0], 128 * E32 * 2 * spread, "mean")
        inside(stats[..., 1], st[..., 1], 300 * E32 * st[..., 1] * (1.0 + spread), "rstd")
        h.close()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_backward(i, dtype):
    shape = SHAPES[i]
    B, P, C, G, pad, sizes = shape
    for act in ACTS:
        print(f"norm backward {shape} {dtype} {act}", flush=True)
        x, gamma, beta, valid, real = inputs(shape, dtype, seed=100 + i)
        if act == "relu":       # u away from the kink, where the statistics' rounding would decide
            x = torch.where(x.abs() < 0.02, torch.full_like(x, 0.5), x)
        dy = make(B, P, C, 0, dtype, 500 + i, 0.5)
        x64, dy64 = behind(x, real, 0.0).double(), behind(dy, real, 0.0).double()
        g64, b64 = gamma.double(), beta.double()
        want, wg, wb, ag, ab = norm_grad(x64, dy64, g64, b64, G, act, EPS, real)
        _, st = norm(x64, g64, b64, G, act, EPS, real)
        xg, dg = padded(behind(x, real, float("nan")), pad), padded(behind(dy, real, float("inf")), pad)
        dx = torch.full((B, P, C + pad), 77.0, dtype=x.dtype, device="cuda")
        dgamma, dbeta = torch.full((C,), 77.0, device="cuda"), torch.full((C,), 77.0, device="cuda")
        h = head().GroupNorm(B, P, C, G, dtype, act, EPS)
        assert h.backward(xg, dg, gamma.cuda(), beta.cuda(), st.float().cuda(), dx[..., :C], dgamma, dbeta,
                          valid) == 0
        kink = torch.zeros_like(x64)
        for b, n in enumerate(real):      # ReLU: a u within rounding of 0 may fall on either side
            if act == "relu" and n:
                u = norm_sample(x64[b, :n], g64, b64, G, "none", EPS)[0]
                kink[b, :n] = (u.abs() < 1e-4).double() * dy64[b, :n].abs()
        rstd = st[..., 1].repeat_interleave(C // G, 1)[:, None, :]
        mean = st[..., 0].repeat_interleave(C // G, 1)[:, None, :]
        xh = ((x64 - mean) * rstd).abs()
        e_xh = 8 * E32 * xh + 2 * E32 * mean.abs() * rstd
        e_du = dy64.abs() * (g64.abs() * e_xh + 16 * E32 * (1.0 + xh)) + kink
        share = (e_du.amax((1, 2)) + 128 * E32 * dy64.abs().amax((1, 2)) * 1.13 * (1 + xh.amax((1, 2))))
        e_sum = (share * g64.abs().max())[:, None, None] * (1.0 + xh.amax((1, 2))[:, None, None])
        bound = rstd * (g64.abs() * e_du + e_sum * (1.0 + xh) + 8 * E32 * (dy64.abs() * 1.13 * g64.abs() + xh))
        keep = torch.zeros_like(x64)
        for b, n in enumerate(real):
            keep[b, :n] = 1.0
        bound = (bound + U[dtype] * (want.abs() + bound)) * keep + TINY[dtype]
        inside(dx[..., :C], want, bound, "dx")
        assert bool((dx[..., C:] == 77.0).all()), "written beyond the rows"
        inside(dgamma, wg, 128 * E32 * ag + ((e_du * xh + dy64.abs() * 1.13 * e_xh) * keep).sum((0, 1)) + 1e-30, "dgamma")
        inside(dbeta, wb, 128 * E32 * ab + (e_du * keep).sum((0, 1)) + 1e-30, "dbeta")
        h.close()


@pytest.mark.parametrize("act", ACTS)
def test_gradient_against_differences(act):
    """<dx, v> + <dgamma, vg> + <dbeta, vb> against the central difference of
    sum(y dy), formed in 64 bits, along random directions."""
    B, P, C, G = 2, 37, 24, 6
    x, gamma, beta, _, real = inputs((B, P, C, G, 0, None), "f32", seed=9)
    dy = make(B, P, C, 0, "f32", 10)
    h = head().GroupNorm(B, P, C, G, "f32", act, EPS)
    _, stats = h.run(x.cuda(), gamma.cuda(), beta.cuda())
    dx, dgamma, dbeta = (t.cpu().double() for t in
                         h.run_backward(x.cuda(), dy.cuda(), gamma.cuda(), beta.cuda(), stats))
    g = torch.Generator().manual_seed(11)
    step = 1e-5
    for _ in range(6):
        v, vg, vb = (torch.randn(s, generator=g, dtype=torch.float64) for s in (x.shape, gamma.shape, beta.shape))

        def loss(t):
            y, _ = norm(x.double() + t * v, gamma.double() + t * vg, beta.double() + t * vb, G, act, EPS, real)
            return float((y * dy.double()).sum())

        slope = (loss(step) - loss(-step)) / (2 * step)
        mine = float((dx * v).sum() + (dgamma * vg).sum() + (dbeta * vb).sum())
        # ReLU: about step * 1.2 |du| of the B P C kinks lie between the two points
        assert abs(mine - slope) <= 1e-4 * max(1.0, abs(slope)) + (0.05 if act == "relu" else 0.0)
    h.close()


def test_mean_far_from_zero():
    """A mean 4000 times the spread: the variance keeps its digits."""
    shape = (2, 3001, 32, 4, 0, None)
    x, gamma, beta, _, real = inputs(shape, "f32", seed=3, scale=0.25, shift=1000.0)
    x64, g64, b64 = x.double(), gamma.double(), beta.double()
    h = head().GroupNorm(2, 3001, 32, 4, "f32", "none", EPS)
    y, stats = h.run(x.cuda(), gamma.cuda(), beta.cuda())
    want, st = norm(x64, g64, b64, 4, "none", EPS, real)
    inside(y, want, bounds_y(x64, g64, b64, 4, "none", real, "f32", want), "y")
    inside(stats[..., 1], st[..., 1], 512 * E32 * st[..., 1], "rstd")
    h.close()


def test_infinities_stay_in_their_group_and_sample():
    x, gamma, beta, _, real = inputs((2, 50, 16, 4, 0, None), "f16", seed=4)
    x[0, 7, 5] = float("inf")
    x[1, 3, 0] = float("nan")
    h = head().GroupNorm(2, 50, 16, 4, "f16", "silu", EPS)
    y, stats = h.run(x.cuda(), gamma.cuda(), beta.cuda())
    y = y.cpu()
    assert bool(y[0, :, 4:8].isnan().all()) and bool(y[1, :, :4].isnan().all())
    assert int(y.isnan().sum()) == 2 * 50 * 4
    h.close()


def test_other_orders_views_and_in_place():
    """Samples and pixels exchanged, [B][H][W][C] maps, y in x's place, dx in
    dy's, no gamma and beta, no stats."""
    B, P, C, G = 3, 20, 32, 4
    x, gamma, beta, _, real = inputs((B, P, C, G, 0, None), "bf16", seed=5)
    h = head().GroupNorm(8, 100, C, G, "bf16", "gelu", EPS)
    y, stats = h.run(x.cuda(), gamma.cuda(), beta.cuda())
    swapped = x.cuda().transpose(0, 1).contiguous().transpose(0, 1)      # pixel stride B C, sample stride C
    out = torch.empty((P, B, C), dtype=x.dtype, device="cuda").transpose(0, 1)
    assert h.forward(swapped, gamma.cuda(), beta.cuda(), out) == 0
    assert torch.equal(out, y)
    image = x.cuda().reshape(B, 4, 5, C)
    y4, _ = h.run(image, gamma.cuda(), beta.cuda())
    assert torch.equal(y4.reshape(B, P, C), y)
    dy = make(B, P, C, 0, "bf16", 6).cuda()
    dx, dgamma, dbeta = h.run_backward(x.cuda(), dy, gamma.cuda(), beta.cuda(), stats)
    over = dy.clone()
    assert h.backward(x.cuda(), over, gamma.cuda(), beta.cuda(), stats, over) == 0
    assert torch.equal(over, dx)
    only = torch.empty(C, device="cuda")
    assert h.backward(x.cuda(), dy, gamma.cuda(), beta.cuda(), stats, dbeta=only) == 0
    assert torch.equal(only, dbeta)
    place = x.cuda().clone()
    assert h.forward(place, gamma.cuda(), beta.cuda(), place) == 0
    assert torch.equal(place, y)
    plain, _ = h.run(x.cuda(), None, None)
    ones, _ = h.run(x.cuda(), torch.ones(C, device="cuda"), torch.zeros(C, device="cuda"))
    assert torch.equal(plain, ones)
    h.close()


@pytest.mark.parametrize("C,P", [(64, 3000), (50, 3000), (32, 100)])
def test_pointers_off_16_bytes_and_large_maps_in_place(C, P):
    """Maps that start one element into their buffers give the same."""
    G = 2
    x, gamma, beta, _, real = inputs((2, P, C, G, 0, None), "f16", seed=8)
    dy = make(2, P, C, 0, "f16", 9).cuda()
    h = head().GroupNorm(2, P, C, G, "f16", "silu", EPS)
    y, stats = h.run(x.cuda(), gamma.cuda(), beta.cuda())

    def off(t):
        full = torch.full(t.shape[:-1] + (C + 1,), 77.0, dtype=t.dtype, device="cuda")
        full[..., 1:] = t
        return full

    place = off(x.cuda())
    assert h.forward(place[..., 1:], gamma.cuda(), beta.cuda(), place[..., 1:]) == 0
    assert torch.equal(place[..., 1:], y) and bool((place[..., 0] == 77.0).all())
    dx, dg, db = h.run_backward(x.cuda(), dy, gamma.cuda(), beta.cuda(), stats)
    place = off(dy)
    dg2, db2 = torch.empty_like(dg), torch.empty_like(db)
    assert h.backward(off(x.cuda())[..., 1:], place[..., 1:], gamma.cuda(), beta.cuda(), stats, place[..., 1:], dg2,
                      db2) == 0
    assert torch.equal(place[..., 1:], dx) and torch.equal(dg, dg2) and torch.equal(db, db2)
    h.close()


def test_nothing_to_do():
    h = head().GroupNorm(2, 10, 8, 2, "f32")
    gamma = torch.ones(8, device="cuda")
    for B, P in ((0, 10), (2, 0)):
        x = torch.empty((B, P, 8), device="cuda")
        stats = torch.zeros((B, 2, 2), device="cuda")
        dg, db = torch.full((8,), 5.0, device="cuda"), torch.full((8,), 5.0, device="cuda")
        assert h.forward(x, gamma, gamma, torch.empty_like(x), stats) == 0
        assert h.backward(x, x, gamma, gamma, stats, torch.empty_like(x), dg, db) == 0
        assert float(dg.abs().max()) == 0.0 and float(db.abs().max()) == 0.0
    h.close()


def test_runs_repeat_and_streams_and_graphs():
    """Two runs agree bit for bit; a side stream and every replay of a graph
    give the eager result, with eager calls in between."""
    B, P, C, G = 2, 5000, 64, 8
    h = head().GroupNorm(B, P, C, G, "f16", "silu", EPS)
    gamma, beta = torch.rand(C, device="cuda") + 0.5, torch.rand(C, device="cuda")
    xs = [make(B, P, C, 0, "f16", 20 + i).cuda() for i in range(3)]
    dys = [make(B, P, C, 0, "f16", 30 + i).cuda() for i in range(3)]

    def eager(i):
        y, stats = h.run(xs[i], gamma, beta)
        return (y, stats) + h.run_backward(xs[i], dys[i], gamma, beta, stats)

    want = [eager(i) for i in range(3)]
    assert all(torch.equal(a, b) for a, b in zip(want[0], eager(0)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = eager(1)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want[1], got))
    x, dy = xs[0].clone(), dys[0].clone()
    y, dx, stats = torch.empty_like(x), torch.empty_like(x), torch.empty((B, G, 2), device="cuda")
    dg, db = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert h.forward(x, gamma, beta, y, stats) == 0
        assert h.backward(x, dy, gamma, beta, stats, dx, dg, db) == 0
    for step in range(6):
        i = step % 3
        x.copy_(xs[i])
        dy.copy_(dys[i])
        for t in (y, dx, stats, dg, db):
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want[i], (y, stats, dx, dg, db))), step
        if step % 2:
            assert all(torch.equal(a, b) for a, b in zip(want[2 - i], eager(2 - i)))
    h.close()


def test_offsets_beyond_32_bits():
    """2,200,000 pixels of 1024 channels: 2.25e9 elements; the rows at the far
    end are those of the same values near the start."""
    P, C, G = 2_200_000, 1024, 32
    x = torch.empty((1, P, C), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    part = torch.randn((1, P // 10, C), generator=g, device="cuda").to(torch.bfloat16)
    for i in range(10):
        x[:, i * (P // 10):(i + 1) * (P // 10)] = part
    gamma, beta = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    h = head().GroupNorm(1, P, C, G, "bf16", "silu", EPS)
    y, stats = h.run(x, gamma, beta)
    tenth, tenth_stats = h.run(part, gamma, beta)
    n = P // 10
    assert torch.equal(y[:, -n:], y[:, :n])
    assert float((stats - tenth_stats).abs().max()) < 1e-5
    assert float((y[:, :n].float() - tenth.float()).abs().max()) <= 2.0 ** -6
    dx, dgamma, dbeta = h.run_backward(x, y, gamma, beta, stats)
    assert torch.equal(dx[:, -n:], dx[:, :n])
    h.close()
