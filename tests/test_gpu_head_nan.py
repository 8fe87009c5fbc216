"""GPU tests of NaNs and infinities in the head operators: they reach what
their definition says and nothing else, in every kind of kernel."""
import pytest

from tests.headref import ACTS, DTYPES

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def head():
    from paper_2609_16874_amd import head as h
    return h


def draw(shape, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(shape, generator=g)).to(DTYPES[dtype]).cuda()


def same_but(got, clean, touched):
    """NaN where touched, otherwise the clean result bit for bit."""
    assert bool(got[touched].isnan().all())
    assert torch.equal(got[~touched], clean[~touched])


#        rows, in, out: few rows; one pass over the rows; tiles, split and staged
LINEAR = [(9, 40, 24), (700, 64, 48), (700, 300, 264), (700, 301, 265)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ACTS[1:])
@pytest.mark.parametrize("M,K,N", LINEAR)
def test_linear_gradient_of_a_nan(M, K, N, act, dtype):
    print(f"linear gradient with a NaN {M} {K} {N} {act} {dtype}", flush=True)
    h = head().Linear(M, K, N, dtype, act)
    x, w, dy, z = (draw(s, dtype, 10 + i, 0.5) for i, s in enumerate(((M, K), (N, K), (M, N), (M, N))))
    clean = h.run_backward(x, w, dy, z)
    z[5, 7] = float("nan")
    dx, dw, db = h.run_backward(x, w, dy, z)
    rows, cols = torch.arange(M, device="cuda") == 5, torch.arange(N, device="cuda") == 7
    same_but(dx, clean[0], rows[:, None].expand(M, K))
    same_but(dw, clean[1], cols[:, None].expand(N, K))
    same_but(db, clean[2], cols)
    h.close()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,K,N", LINEAR)
def test_linear_forward_of_a_nan_or_an_infinity(M, K, N, dtype, bad):
    """ReLU, so that an infinity stays one: its row is what 64 bits say."""
    print(f"linear forward with {bad} {M} {K} {N} {dtype}", flush=True)
    h = head().Linear(M, K, N, dtype, "relu")
    x, w = draw((M, K), dtype, 20, 0.5), draw((N, K), dtype, 21)
    w[w == 0] = 1.0
    clean = h.run(x, w)
    x[5, 7] = bad
    y = h.run(x, w)
    rest = torch.arange(M, device="cuda") != 5
    assert torch.equal(y[rest], clean[rest])
    z = x[5].double() @ w.double().t()
    want = torch.where(z < 0, torch.zeros_like(z), z)
    assert torch.equal(y[5].isnan(), want.isnan()) and torch.equal(y[5].isinf(), want.isinf())
    h.close()


#        B, P, C, G: one pass; two passes, vectors within groups, across them, across rows' ends; past the caches
NORM = [(2, 50, 16, 4), (2, 9001, 64, 8), (2, 9001, 64, 16), (2, 9001, 50, 5), (2, 300_000, 64, 4)]


def group_of(shape, b, c):
    """The map's places in channel c's group of sample b."""
    B, P, C, G = shape
    out = torch.zeros((B, P, C), dtype=torch.bool, device="cuda")
    cpg = C // G
    out[b, :, c // cpg * cpg:(c // cpg + 1) * cpg] = True
    return out


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", NORM)
def test_norm_forward_of_a_nan_or_an_infinity(shape, dtype, bad):
    """At the first pixel, a middle one and the last: the group of that sample
    is NaN, the rest is as without."""
    B, P, C, G = shape
    print(f"norm forward with {bad} {shape} {dtype}", flush=True)
    h = head().GroupNorm(B, P, C, G, dtype, "relu")
    x = draw((B, P, C), dtype, 30)
    clean, clean_stats = h.run(x, None, None)
    for p in (0, P // 2, P - 1):
        hurt = x.clone()
        hurt[1, p, C - 2] = bad
        y, stats = h.run(hurt, None, None)
        same_but(y, clean, group_of(shape, 1, C - 2))
        g = (C - 2) // (C // G)
        assert bool(stats[1, g, 1].isnan())
        keep = torch.ones((B, G), dtype=torch.bool, device="cuda")
        keep[1, g] = False
        assert torch.equal(stats[keep], clean_stats[keep])
    h.close()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("shape", NORM)
def test_norm_gradient_of_a_nan(shape, act, dtype):
    """A NaN in x (beside statistics without one) and one in dy: dx is NaN in
    that sample's group, dgamma and dbeta in that channel, except that x does
    not enter dbeta without an activation."""
    B, P, C, G = shape
    print(f"norm gradient with a NaN {shape} {act} {dtype}", flush=True)
    h = head().GroupNorm(B, P, C, G, dtype, act)
    x, dy = draw((B, P, C), dtype, 40), draw((B, P, C), dtype, 41, 0.1)
    _, stats = h.run(x, None, None)
    clean = h.run_backward(x, dy, None, None, stats)
    channel = torch.arange(C, device="cuda") == C - 2
    for which in (0, 1):
        hurt = [x.clone(), dy.clone()]
        hurt[which][1, P // 3, C - 2] = float("nan")
        dx, dgamma, dbeta = h.run_backward(*hurt, None, None, stats)
        same_but(dx, clean[0], group_of(shape, 1, C - 2))
        same_but(dgamma, clean[1], channel)
        same_but(dbeta, clean[2], channel & (which == 1 or act != "none"))
    h.close()
