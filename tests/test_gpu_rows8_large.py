"""GPU test of the weight's gradient from rows in 8 bits whose offsets pass 32 bits."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N", [16, 136, 264])
@pytest.mark.parametrize("act", ["none", "relu"])
def test_weight_gradient_beyond_32_bits(N, act):
    """4,500,000 rows of 1024 bytes, ten times the same 450,000, so a row that is
    read 2^32 bytes too early is another one.  Bytes, scales that are powers of two
    and dy of 0 and +-1 make every product a multiple of 1/2 that 16 bits hold; the
    sums of their sizes stay below 2^23, so sums in binary32 are exact in any order,
    and dw is the 64-bit sum rounded once."""
    from paper_2609_16874_amd import head
    M, K, parts = 4_500_000, 1024, 10
    n = M // parts
    g = torch.Generator(device="cuda").manual_seed(N)

    def whole(lo, hi, *shape):
        return torch.randint(lo, hi, shape, device="cuda", generator=g)

    part = whole(-127, 128, n, K).to(torch.int8)
    s_part = torch.exp2(whole(-1, 2, n).float())
    dy_part = ((whole(0, 64, n, N) == 0) * (2 * whole(0, 2, n, N) - 1)).to(torch.bfloat16)
    z_part = whole(-127, 128, n, N).to(torch.int8)
    q, s, dy = part.repeat(parts, 1), s_part.repeat(parts), dy_part.repeat(parts, 1)
    kept = (z_part.repeat(parts, 1), torch.full((M,), 0.01, device="cuda")) if act == "relu" else (None, None)
    dw, db = torch.empty((N, K), dtype=torch.bfloat16, device="cuda"), torch.empty(N, device="cuda")
    w = torch.ones((N, K), dtype=torch.bfloat16, device="cuda")
    lin = head.Linear(M, K, N, "bf16", act)
    assert lin.backward8(q, s, w, dy, *kept, dweight=dw, dbias=db) == 0
    torch.cuda.synchronize()
    lin.close()
    dz = dy_part.double() * (z_part > 0 if act == "relu" else 1.0)
    x, dzt = part.double() * s_part.double()[:, None], dz.t().contiguous()
    want, mag = parts * (dzt @ x), parts * (dzt.abs() @ x.abs())
    assert float(mag.max()) < 2.0 ** 23
    assert torch.equal(dw, want.to(torch.bfloat16))
    assert torch.equal(db.double(), parts * dz.sum(0))
