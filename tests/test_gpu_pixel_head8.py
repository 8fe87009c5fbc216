"""GPU tests of the head served in 8-bit integers (PixelHead8) on parameters
that are neither 1 nor 0."""
import pytest

from tests.headref import E32, TINY, U
from tests.rows8ref import values

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

H, W, C, G, D = 25, 33, 48, 8, 16


def heads(dtype, blocks):
    """A head with parameters of its own, and the one that serves it."""
    from paper_2609_16874_amd.pixel_head import PixelHead, PixelHead8
    h = PixelHead(H, W, C, G, D, dtype, "gelu", seed=3, blocks=blocks)
    g = torch.Generator().manual_seed(4)
    for k, v in h.params.items():
        if "w_" not in k:
            v += 0.3 * torch.randn(v.shape, generator=g).cuda()
    x = torch.randn((H, W, C), generator=g).to(h.params["w_emb"].dtype).cuda()
    return h, PixelHead8(h), x


def near_rows(packed, w):
    """Rows in 8 bits against what was packed: half a step of 1/127 of a row's
    largest value, and a rounding."""
    got, w = values(*(t.cpu() for t in packed)), w.cpu().double()
    step = w.abs().amax(1, keepdim=True) / 127.0
    assert bool(((got - w).abs() <= (0.5 + 2.0 ** -15) * step).all())


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("blocks", [0, 2])
def test_outputs_are_its_operators_one_after_another(blocks, dtype):
    """From the rows that each step had, in 64 bits.  A product's sum is exact; its
    value is off by 3 e for the conversion and the scales and e for the bias, e =
    2^-24, and a rounding to the type."""
    from paper_2609_16874_amd import rows8
    trained, served, x = heads(dtype, blocks)
    p = trained.params
    emb, fg = served.forward(x)
    assert emb.shape == (H, W, D) and fg.shape == (H, W) and emb.dtype is x.dtype
    rows, stream = x.reshape(H * W, C), None
    for b in served.blocks:
        rows, stream = b.forward(rows, stream)
    if blocks:
        rows = rows + stream
    hidden, _ = trained.norm.run(rows.view(1, H, W, C), p["gamma"], p["beta"])
    kept = values(*(t.cpu() for t in rows8.packed(hidden.view(H * W, C))))
    for got, w8, weight, bias in ((emb.reshape(-1, D), served.w_emb, p["w_emb"], p["b_emb"]),
                                  (fg.reshape(-1, 1), served.w_fg, p["w_fg"], p["b_fg"])):
        near_rows(w8, weight)
        dot = kept @ values(*(t.cpu() for t in w8)).t()
        want = dot + bias.cpu().double()
        off = 4 * E32 * (dot.abs() + want.abs())
        far = (got.cpu().double() - want).abs() - (off + U[dtype] * (want.abs() + off) + TINY[dtype])
        assert float(far.max()) <= 0.0
    for b, t in zip(served.blocks, trained.blocks):
        near_rows(b.w_up, t.params["w_up"])
        near_rows(b.w_down, t.params["w_down"])
        assert all(torch.equal(getattr(b, k), t.params[k]) for k in ("gamma", "b_up", "b_down"))
    served.close()
    trained.close()


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("blocks", [0, 2])
def test_outputs_are_near_the_trained_heads(blocks, dtype):
    """A rounding to a row's steps is off by max / (127 sqrt 12), which for rows
    whose largest value is up to 4.4 times their mean square's root is 1 % of it.  A
    product of two such operands is off by 1.5 %, and of a sum with a bias by no
    more.  Two blocks of two products each and the projection after them, each
    passing on what came before: sqrt(5) 1.5 % = 3.4 %, of which the group norm and
    GELU, whose slopes are near 1, make three times that at most: 10 %."""
    trained, served, x = heads(dtype, blocks)
    for got, want in zip(served.forward(x), trained.forward(x)):
        got, want = got.double(), want.double()
        assert float((got - want).norm()) <= 0.1 * float(want.norm())
    # what was trained afterwards does not reach a head that is served already
    before = [t.clone() for t in served.forward(x)]
    for v in trained.params.values():
        v.zero_()
    assert all(torch.equal(a, b) for a, b in zip(served.forward(x), before))
    served.close()
    trained.close()
