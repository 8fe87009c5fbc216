"""GPU test of the pixel head: its gradients against 64-bit autograd, and a
short training run whose outputs the decoder then reads."""
import pytest

from tests.headref import norm_sample

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_gradients_match_autograd():
    """fp32, so that the head's own rounding stays far below the bound: 2e-5 of
    each gradient's largest value (sums of up to 315 terms of order 1)."""
    from paper_2609_16874_amd.pixel_head import PixelHead
    H, W, C, G, D = 15, 21, 24, 4, 16
    h = PixelHead(H, W, C, G, D, "f32", "gelu", seed=3)
    g = torch.Generator().manual_seed(4)
    x, d_emb, d_fg = (torch.randn(s, generator=g) for s in ((H, W, C), (H, W, D), (H, W)))
    h.params["gamma"] += 0.3 * torch.randn(C, generator=g).cuda()
    h.params["beta"] += 0.3 * torch.randn(C, generator=g).cuda()
    emb, fg = h.forward(x.cuda())
    got = h.backward(d_emb.cuda(), d_fg.cuda())
    p = {k: v.cpu().double().requires_grad_(True) for k, v in h.params.items()}
    x64 = x.double().requires_grad_(True)
    y, _, _ = norm_sample(x64.reshape(-1, C), p["gamma"], p["beta"], G, "gelu", 1e-5)
    e, f = y @ p["w_emb"].t() + p["b_emb"], y @ p["w_fg"].t() + p["b_fg"]
    loss = (e * d_emb.double().reshape(-1, D)).sum() + (f[:, 0] * d_fg.double().reshape(-1)).sum()
    loss.backward()
    assert float((emb.cpu().double() - e.detach().reshape(H, W, D)).abs().max()) < 1e-5
    assert float((fg.cpu().double() - f.detach().reshape(H, W)).abs().max()) < 1e-5
    want = {k: v.grad for k, v in p.items()}
    want["features"] = x64.grad
    for k, v in want.items():
        far = float((got[k].cpu().double().reshape(v.shape) - v).abs().max())
        assert far <= 2e-5 * max(1.0, float(v.abs().max())), (k, far)
    h.close()


def test_training_makes_the_frame_decodable():
    from paper_2609_16874_amd import pixel_head
    losses, before, after = pixel_head.main(config=1, steps=60)
    assert losses[-1] < 0.1 * losses[0]
    assert after[1] > before[1] and after[1] > 0.8
