"""GPU tests of the head operators on large data: maps that are written past
the caches, and offsets beyond 32 bits, against their definition in 64 bits.

The bounds of the norm are those of the smaller maps (test_gpu_head_norm.py:
e = 2^-24, chains of at most 128 additions), which hold for the maps past the
caches: a thread walks at most 40 rows of them.  At 2,200,000 pixels a thread
walks 1074 rows, and its values lie about its first one: the mean is off by
less than 2400 e max|x - mean|, and the sums of squares, which are then twice
the variance's on average and enter twice, leave rstd within 4000 e.

The products take small whole numbers, whose sums are exact in binary32: every
output is the exact one rounded once, whatever the order of the sums."""
import pytest

from tests.headref import DTYPES, E32, TINY, U, activation, activation_grad, norm_sample

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
EPS = 1e-5


def head():
    from paper_2609_16874_amd import head as h
    return h


def within(got, want, bound, what):
    got = got.double()
    assert got.shape == want.shape and not bool(got.isnan().any()), what
    far = float(((got - want).abs() - bound).max())
    assert far <= 0.0, f"{what}: {far:.3g} beyond its bound"


def placed(m, place):
    """The map with its rows one after another, in a wider buffer, or off by an element."""
    C = m.shape[-1]
    before, behind = {"apart": (0, 0), "in place": (0, 0), "padded": (0, 8), "off": (1, 0)}[place]
    full = torch.full(m.shape[:-1] + (before + C + behind,), 77.0, dtype=m.dtype, device="cuda")
    full[..., before:before + C] = m
    return full, full[..., before:before + C]


def untouched(full, C, place):
    rest = full[..., C:] if place != "off" else full[..., :1]
    return bool((rest == 77.0).all())


@pytest.mark.parametrize("place", ["apart", "padded", "off", "in place"])
@pytest.mark.parametrize("dtype,C,G,act", [("f16", 64, 8, "silu"), ("bf16", 96, 32, "gelu"), ("f32", 64, 16, "silu"),
                                           ("f32", 64, 32, "gelu")])
def test_maps_past_the_caches(dtype, C, G, act, place):
    """Three samples, one empty and one ragged, of 147 MB or more read and
    written; vectors within a group and across groups."""
    print(f"maps past the caches {dtype} {C} {G} {act} {place}", flush=True)
    B, size = 3, 4 if dtype == "f32" else 2
    P = (148 << 20) // (2 * B * C * size) | 1
    sizes = (P, 0, P * 3 // 4 + 1)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = (1.5 * torch.randn((B, P, C), generator=g, device="cuda")
         + 0.5 * torch.randn(C, generator=g, device="cuda")).to(DTYPES[dtype])
    dy = (0.5 * torch.randn((B, P, C), generator=g, device="cuda")).to(DTYPES[dtype])
    gamma = 1.0 + 0.3 * torch.randn(C, generator=g, device="cuda")
    beta = 0.3 * torch.randn(C, generator=g, device="cuda")
    valid = torch.tensor(sizes, dtype=torch.int32, device="cuda")
    for b, n in enumerate(sizes):
        x[b, n:] = dy[b, n:] = float("nan")
    h = head().GroupNorm(B, P, C, G, dtype, act, EPS)
    _, px = placed(x, place)
    full, y = placed(torch.full_like(x, 77.0), place)
    if place == "in place":
        y = px
    stats = torch.full((B, G, 2), 77.0, device="cuda")
    assert h.forward(px, gamma, beta, y, stats, valid) == 0
    assert place == "in place" or untouched(full, C, place)
    exact = torch.zeros((B, G, 2), dtype=torch.float64, device="cuda")
    exact[..., 1] = EPS ** -0.5
    cpg = C // G
    g64, b64 = gamma.double(), beta.double()
    for b, n in enumerate(sizes):
        assert bool((y[b, n:] == 0.0).all()), "pixels behind a sample's are 0"
        if n == 0:
            continue
        x64 = x[b, :n].double()
        want, mean, rstd = norm_sample(x64, g64, b64, G, act, EPS)
        exact[b, :, 0], exact[b, :, 1] = mean, rstd
        m, r = mean.repeat_interleave(cpg), rstd.repeat_interleave(cpg)
        spread = (x64 - m).abs().amax(0).reshape(G, -1).amax(1).repeat_interleave(cpg)
        xh = ((x64 - m) * r).abs()
        e_xh = r * (128 * E32 * spread + 2 * E32 * m.abs()) + (256 + 6) * E32 * xh
        u = xh * g64.abs() + b64.abs()
        bound = 1.13 * (g64.abs() * e_xh + 2 * E32 * u) + 16 * E32 * (u + 1.0)
        within(y[b, :n], want, bound + U[dtype] * (want.abs() + bound) + TINY[dtype], f"y of sample {b}")
    within(stats[..., 0], exact[..., 0], 128 * E32 * 8.0, "mean")
    within(stats[..., 1], exact[..., 1], 256 * E32 * exact[..., 1], "rstd")
    del y, full, px

    _, px = placed(x, place)
    _, pd = placed(dy, place)
    full, dx = placed(torch.full_like(x, 77.0), place)
    if place == "in place":
        dx = pd
    dgamma, dbeta = torch.full_like(gamma, 77.0), torch.full_like(beta, 77.0)
    assert h.backward(px, pd, gamma, beta, exact.float(), dx, dgamma, dbeta, valid) == 0
    assert place == "in place" or untouched(full, C, place)
    wg, wb, eg, eb = (torch.zeros(C, dtype=torch.float64, device="cuda") for _ in range(4))
    for b, n in enumerate(sizes):
        assert bool((dx[b, n:] == 0.0).all())
        if n == 0:
            continue
        x64, d64 = x[b, :n].double(), dy[b, :n].double()
        m, r = (exact[b, :, i].repeat_interleave(cpg) for i in (0, 1))
        xh = (x64 - m) * r
        du = d64 * activation_grad(act, xh * g64 + b64)
        a = (du * g64).reshape(n, G, cpg).mean((0, 2)).repeat_interleave(cpg)
        q = (du * g64 * xh).reshape(n, G, cpg).mean((0, 2)).repeat_interleave(cpg)
        want = r * (du * g64 - a - xh * q)
        ax, ad = xh.abs(), d64.abs()
        e_xh = 8 * E32 * ax + 2 * E32 * m.abs() * r
        e_du = ad * (g64.abs() * e_xh + 16 * E32 * (1.0 + ax))
        share = e_du.max() + 128 * E32 * ad.max() * 1.13 * (1.0 + ax.max())
        e_sum = share * g64.abs().max() * (1.0 + ax.max())
        bound = r * (g64.abs() * e_du + e_sum * (1.0 + ax) + 8 * E32 * (ad * 1.13 * g64.abs() + ax))
        within(dx[b, :n], want, bound + U[dtype] * (want.abs() + bound) + TINY[dtype], f"dx of sample {b}")
        wg += (du * xh).sum(0)
        wb += du.sum(0)
        eg += 128 * E32 * (du * xh).abs().sum(0) + (e_du * ax + ad * 1.13 * e_xh).sum(0)
        eb += 128 * E32 * du.abs().sum(0) + e_du.sum(0)
    within(dgamma, wg, eg, "dgamma")
    within(dbeta, wb, eb, "dbeta")
    h.close()


def test_norm_offsets_beyond_32_bits_against_the_definition():
    """2,200,000 pixels of 1024 channels: 2.25e9 elements, every one checked."""
    P, C, G, parts = 2_200_000, 1024, 32, 10
    n, cpg = P // parts, C // G
    x, dy = (torch.empty((1, P, C), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(1)
    for i in range(parts):
        x[0, i * n:(i + 1) * n] = torch.randn((n, C), generator=g, device="cuda")
        dy[0, i * n:(i + 1) * n] = 0.5 * torch.randn((n, C), generator=g, device="cuda")
    gamma, beta = 1.0 + 0.3 * torch.randn(C, generator=g, device="cuda"), torch.randn(C, generator=g, device="cuda")
    h = head().GroupNorm(1, P, C, G, "bf16", "silu", EPS)
    y, stats = h.run(x, gamma, beta)
    g64, b64 = gamma.double(), beta.double()

    def chunks(t):
        return ((i, t[0, i * n:(i + 1) * n].double()) for i in range(parts))

    mean = sum(v.reshape(n, G, cpg).sum((0, 2)) for _, v in chunks(x)) / (P * cpg)
    square = sum((v.reshape(n, G, cpg) - mean[:, None]).pow(2).sum((0, 2)) for _, v in chunks(x)) / (P * cpg)
    rstd = (square + EPS).rsqrt()
    m, r = mean.repeat_interleave(cpg), rstd.repeat_interleave(cpg)
    within(stats[0, :, 0], mean, 2400 * E32 * 8.0, "mean")
    within(stats[0, :, 1], rstd, 4000 * E32 * rstd, "rstd")
    stats = torch.stack((mean, rstd), -1)[None].float()
    dx, dgamma, dbeta = h.run_backward(x, dy, gamma, beta, stats)
    wg, wb, ag, ab, eg, eb = (torch.zeros(C, dtype=torch.float64, device="cuda") for _ in range(6))
    most = 0.0
    for i, v in chunks(x):
        xh = (v - m) * r
        want = activation("silu", xh * g64 + b64)
        u, ax = xh.abs() * g64.abs() + b64.abs(), xh.abs()
        spread = (v - m).abs().max()
        e_xh = r * (2400 * E32 * spread + 2 * E32 * m.abs()) + (4000 + 6) * E32 * ax
        bound = 1.13 * (g64.abs() * e_xh + 2 * E32 * u) + 16 * E32 * (u + 1.0)
        within(y[0, i * n:(i + 1) * n], want, bound + U["bf16"] * (want.abs() + bound), f"y of part {i}")
        d64 = dy[0, i * n:(i + 1) * n].double()
        du = d64 * activation_grad("silu", xh * g64 + b64)
        e_xh = 8 * E32 * ax + 2 * E32 * m.abs() * r
        e_du = d64.abs() * (g64.abs() * e_xh + 16 * E32 * (1.0 + ax))
        most = max(most, float(e_du.max() + 1200 * E32 * d64.abs().max() * 1.13 * (1.0 + ax.max())), )
        wg += (du * xh).sum(0)
        wb += du.sum(0)
        ag += (du * xh).abs().sum(0)
        ab += du.abs().sum(0)
        eg += (e_du * ax + d64.abs() * 1.13 * e_xh).sum(0)
        eb += e_du.sum(0)
    within(dgamma, wg, 1200 * E32 * ag + eg, "dgamma")
    within(dbeta, wb, 1200 * E32 * ab + eb, "dbeta")
    a = (wb * g64).reshape(G, cpg).sum(1).repeat_interleave(cpg) / (P * cpg)
    q = (wg * g64).reshape(G, cpg).sum(1).repeat_interleave(cpg) / (P * cpg)
    for i, v in chunks(x):
        xh, d64 = (v - m) * r, dy[0, i * n:(i + 1) * n].double()
        ax = xh.abs()
        want = r * (d64 * activation_grad("silu", xh * g64 + b64) * g64 - a - xh * q)
        e_du = d64.abs() * (g64.abs() * (8 * E32 * ax + 2 * E32 * m.abs() * r) + 16 * E32 * (1.0 + ax))
        e_sum = most * g64.abs().max() * (1.0 + ax.max())
        bound = r * (g64.abs() * e_du + e_sum * (1.0 + ax) + 8 * E32 * (d64.abs() * 1.13 * g64.abs() + ax))
        within(dx[0, i * n:(i + 1) * n], want, bound + U["bf16"] * (want.abs() + bound), f"dx of part {i}")
    h.close()


def whole_numbers(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-2, 3, shape, generator=g, dtype=torch.int8, device="cuda").to(DTYPES[dtype])


@pytest.mark.parametrize("M,K,N,dtype", [
    (4_400_000, 512, 16, "bf16"),       # narrow product, the gradient in one pass
    (17_000_000, 128, 20, "f16"),       # narrow product, narrow dx and a tiled dw
    (17_000_000, 128, 12, "f32"),       # the same in 32 bits
    (2_200_000, 1024, 136, "bf16"),     # tiles
])
def test_linear_offsets_beyond_32_bits_against_the_definition(M, K, N, dtype):
    """2.2e9 elements of x, every output checked."""
    print(f"linear beyond 32 bits {M} {K} {N} {dtype}", flush=True)
    assert M * K > 2 ** 31
    h = head().Linear(M, K, N, dtype)
    x, w, dy = whole_numbers((M, K), dtype, 1), whole_numbers((N, K), dtype, 2), whole_numbers((M, N), dtype, 3)
    y = h.run(x, w)
    dx, dw, db = h.run_backward(x, w, dy)
    w64 = w.double()
    dw64, db64 = torch.zeros((N, K), dtype=torch.float64, device="cuda"), torch.zeros(N, dtype=torch.float64,
                                                                                      device="cuda")
    step = M // 20
    for lo in range(0, M, step):
        x64, d64 = x[lo:lo + step].double(), dy[lo:lo + step].double()
        assert torch.equal(y[lo:lo + step], torch.mm(x64, w64.t().contiguous()).to(DTYPES[dtype])), lo
        assert torch.equal(dx[lo:lo + step], torch.mm(d64, w64).to(DTYPES[dtype])), lo
        dw64 += torch.mm(d64.t().contiguous(), x64)
        db64 += d64.sum(0)
    assert float(dw64.abs().max()) < 2 ** 24 and float(dw64.abs().max()) > 0.0
    assert torch.equal(dw, dw64.to(DTYPES[dtype]))
    assert torch.equal(db.double(), db64)
    h.close()
