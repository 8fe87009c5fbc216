"""GPU tests of the integer product in tiles of 256 x 256 whose outputs are rows
of whole cache lines (16 bits, strides that are multiples of 64 elements), which
are stored past the caches: whole tiles, tiles that end inside the rows or the
columns, strides longer than the rows, with and without the residual and the
value before the activation.

Bounds as in the tests of the other forms.  e = 2^-24, u the type's half unit:
the whole-number sum is exact (and so is its restatement, a product of whole
numbers in 64 bits), z is off by 3 e |acc s t| for the conversion and two scales
and e |z| for the bias, an activation has a slope of at most 1.13 and adds 16 e
(|z| + 1), the residual e (|y| + 1), and the output's rounding u |y|.  The
reference is computed on the GPU, in 64 bits."""
import pytest

from tests.headref import ACTS, DTYPES, E32, TINY, U, activation
from tests.rows8ref import byte_rows, matrix, target, untouched

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

#        rows, in, out, pad: 256 x 256 tiles fill the chip in one round, 128 x 128 ones in two
SHAPES = [
    (4096, 256, 4096, 0),       # whole tiles, two steps of k
    (4096, 16, 4096, 0),        # a step that k does not fill
    (4000, 528, 3840, 64),      # rows end inside a tile; five steps; lines between the rows
    (3900, 208, 3904, 0),       # rows and columns do
    (3841, 128, 3850, 54),      # one row in the last tiles, columns that end inside a vector
]


def rows8():
    from paper_2609_16874_amd import rows8 as r
    return r


def within(got, want, bound, what):
    far = float(((got.double() - want).abs() - bound).max())
    assert far <= 0.0, f"{what}: {far:.3g} beyond its bound"


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_forward(i, dtype):
    M, K, N, pad = SHAPES[i]
    q, s = (t.cuda() for t in byte_rows(M, K, i, whole_range=i % 2 == 1))
    w, t = (v.cuda() for v in byte_rows(N, K, 100 + i, K ** -0.5))
    if i % 2 == 1:
        s = s / 64
    bias, res = matrix(1, N, "f32", 200 + i)[0].cuda(), matrix(M, N, dtype, 300 + i).cuda()
    dot = (q.double() @ w.double().t()) * s.double()[:, None] * t.double()
    for act in ACTS:
        h = rows8().Linear8(M, K, N, dtype, act)
        for with_res, keep in ((False, False), (True, False), (False, True), (True, True)):
            print(f"wide linear8 {SHAPES[i]} {dtype} {act} residual {with_res} preact {keep}", flush=True)
            (fy, y), (fz, z) = target(M, N, pad, dtype), target(M, N, pad, dtype)
            assert y.stride(0) % 64 == 0 and y.data_ptr() % 128 == 0 and z.data_ptr() % 128 == 0
            r = res if with_res else None
            assert h.forward(q, s, w, t, bias if keep else None, y, r, z if keep else None) == 0
            want_z = dot + bias.double() if keep else dot
            e_z = 4 * E32 * (dot.abs() + want_z.abs())
            want = activation(act, want_z)
            e_y = 1.13 * e_z + 16 * E32 * (want_z.abs() + 1.0) * (act != "none")
            if with_res:
                want = want + res.double()
                e_y = e_y + E32 * (want.abs() + 1.0)
            if keep:
                within(z, want_z, e_z + U[dtype] * (want_z.abs() + e_z) + TINY[dtype], "z")
                assert untouched(fz, z), "written beyond the rows of z"
            within(y, want, e_y + U[dtype] * (want.abs() + e_y) + TINY[dtype], "y")
            assert untouched(fy, y), "written beyond the rows"
            again = torch.empty((M, N), dtype=DTYPES[dtype], device="cuda")
            assert h.forward(q, s, w, t, bias if keep else None, again, r) == 0 and torch.equal(again, y)
        h.close()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_residual_in_place(i, dtype):
    M, K, N, pad = SHAPES[i]
    q, s, w, t = (v.cuda() for v in byte_rows(M, K, 1) + byte_rows(N, K, 2, 0.1))
    h = rows8().Linear8(M, K, N, dtype, "gelu")
    full, over = target(M, N, pad, dtype)
    over.copy_(matrix(M, N, dtype, 3))
    y, z = h.run(q, s, w, t, residual=over, keep=True)
    kept = torch.empty_like(z)
    assert h.forward(q, s, w, t, None, over, residual=over, preact=kept) == 0
    assert torch.equal(over, y) and torch.equal(kept, z) and untouched(full, over)
    h.close()


def test_replays_of_a_graph():
    """Captured once, replayed on other rows, with eager calls in between."""
    M, K, N = 4096, 256, 4096
    qs = [[v.cuda() for v in byte_rows(M, K, 10 + i)] for i in range(3)]
    w, t = (v.cuda() for v in byte_rows(N, K, 1, K ** -0.5))
    res = matrix(M, N, "bf16", 5).cuda()
    h = rows8().Linear8(M, K, N, "bf16", "silu")
    want = [h.run(*v, w, t, residual=res, keep=True) for v in qs]
    q, s, y, z = qs[0][0].clone(), qs[0][1].clone(), torch.empty_like(res), torch.empty_like(res)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert h.forward(q, s, w, t, None, y, residual=res, preact=z) == 0
    for step in range(6):
        i = step % 3
        q.copy_(qs[i][0])
        s.copy_(qs[i][1])
        y.fill_(7)
        z.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[i][0]) and torch.equal(z, want[i][1]), step
        if step % 2:
            assert torch.equal(h.run(*qs[2 - i], w, t, residual=res), want[2 - i][0])
    h.close()
