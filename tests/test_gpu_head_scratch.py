"""GPU tests of the matrix product's scratch: a handle holds what its calls can
use, and its size changes no result."""
import pytest

from tests.headref import DTYPES

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def head():
    from paper_2609_16874_amd import head as h
    return h


def size(*args):
    h = head().Linear(*args)
    n = h.workspace_bytes()
    h.close()
    return n


def test_handles_hold_what_their_calls_can_use():
    """One row: no more than two splits of its product would take, 8 KB.
    The 640 x 640 projection's gradient in one pass: 256 partial dw of 64 x 256
    floats (16.8 MB) and their 262 KB of sums, no dz.  A product whose k is too
    short for splits and that has no activation: dw's splits and sums alone."""
    assert size(1, 1024, 1024, "f16", "silu") <= 16 << 10
    assert size(64, 64, 64, "f32", "gelu") == 0
    assert size(640 * 640, 256, 64, "f16", "silu") <= 256 * 64 * 256 * 4 + (1 << 20)
    # with dz: 7744 x 4096 in 16 bits, no more than 32 MiB of splits and 8 MiB of sums beside it
    dz = 7744 * 4096 * 2
    assert dz <= size(7744, 1024, 4096, "bf16", "gelu") <= dz + (40 << 20) + 1024
    assert size(7744, 1024, 4096, "bf16", "none") <= (40 << 20) + 1024


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,K,N", [(1, 1024, 1024), (65, 2048, 136), (200, 1024, 1024), (400, 700, 760),
                                   (400, 520, 4104), (1500, 1024, 64), (700, 64, 48), (64, 1000, 264), (130, 4096, 72)])
def test_the_size_of_a_handle_changes_no_result(M, K, N, dtype):
    """A handle for M rows and one for many more."""
    print(f"scratch of {M} {K} {N} {dtype}", flush=True)
    g = torch.Generator().manual_seed(1)
    x, w, dy = (torch.randn(s, generator=g).to(DTYPES[dtype]).cuda() for s in ((M, K), (N, K), (M, N)))
    outs = []
    for rows in (M, 100_000):
        h = head().Linear(rows, K, N, dtype, "silu")
        y, z = h.run(x, w, keep=True)
        outs.append((y, z) + h.run_backward(x, w, dy, z))
        torch.cuda.synchronize()
        h.close()
    assert all(torch.equal(a, b) for a, b in zip(*outs))
