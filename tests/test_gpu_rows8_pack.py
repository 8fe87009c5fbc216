"""GPU tests of rows packed into 8 bits and back (cpe_rows8_pack, _unpack).

The scale and the quotients that are rounded to bytes are single divisions of
binary32 values: exactly what torch's division gives.  The values that the bytes stand for are one product of binary32, rounded once
more to the type: exactly what torch's elementwise product and conversion give."""
import pytest

from tests.headref import DTYPES
from tests.rows8ref import LEAST, check_packed, matrix, padded, target, untouched

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

#        rows, width, pad, lead
SHAPES = [
    (1, 1, 0, 0), (1, 3, 0, 0), (7, 5, 2, 1), (5, 8, 0, 0), (9, 9, 0, 3), (40, 63, 1, 0), (33, 64, 0, 0), (300, 65, 3, 1),
    (17, 100, 0, 0), (1000, 127, 0, 0), (129, 256, 8, 0), (64, 511, 0, 0), (3000, 512, 0, 0), (10, 1001, 3, 2),
    (2, 2049, 0, 0), (65, 4096, 0, 0), (3, 4104, 0, 1), (4, 8191, 0, 0), (5, 10000, 24, 0), (2, 16384, 0, 0), (3, 16391, 0, 0),
    (2, 40001, 0, 0), (1, 65536, 0, 0), (70001, 24, 0, 0), (30000, 260, 4, 0),
    (1500, 2500, 0, 0), (900, 4100, 8, 0), (700, 7000, 0, 1), (600, 9000, 0, 0),    # (several turns of a workgroup per row)
]


def rows8():
    from paper_2609_16874_amd import rows8 as r
    return r


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_pack_and_unpack(i, dtype):
    M, C, pad, lead = SHAPES[i]
    x = matrix(M, C, dtype, i) * torch.exp(2.0 * torch.randn((M, 1), generator=torch.Generator().manual_seed(i)))
    x = x.to(DTYPES[dtype])
    fq, q = target(M, C, pad, "i8", lead)
    scale = torch.full((M + 1,), 77.0, device="cuda")
    assert rows8().pack(padded(x, pad, lead), q, scale[:M]) == 0
    check_packed(q, scale[:M], x.double(), 0.0)
    assert torch.equal(scale[:M].cpu(), (x.float().abs().amax(1) / 127.0).clamp(min=LEAST))
    assert torch.equal(q.cpu(), torch.round(x.float() / scale[:M].cpu()[:, None]).to(torch.int8))
    assert untouched(fq, q) and float(scale[M]) == 77.0
    for to in ("f32", "f16", "bf16"):
        fv, v = target(M, C, pad, to, lead)
        assert rows8().unpack(q, scale[:M], v) == 0
        assert torch.equal(v, (q.float() * scale[:M, None]).to(DTYPES[to])), to
        assert untouched(fv, v)


@pytest.mark.parametrize("width", [3, 24, 100, 1000, 5000])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_rows_of_extreme_values(dtype, width):
    """Zeros, one value, NaNs, infinities, the largest and smallest values:
    each row is what it is, whatever its neighbours are."""
    t = DTYPES[dtype]
    x = matrix(12, width, dtype, 5)
    x[1] = 0.0
    x[2] = 0.0
    x[2, width - 1] = 3.0
    x[3, width // 2] = float("nan")
    x[4, 0] = float("inf")
    x[5, width - 1] = float("-inf")
    x[6] = torch.finfo(t).max
    x[7] = -torch.finfo(t).max
    x[8] = torch.finfo(t).smallest_normal
    x[9] = torch.tensor(2.0 ** -149 if dtype == "f32" else 0.0).to(t)
    x[10, 0] = -0.0
    q, scale = rows8().packed(x.cuda())
    back = rows8().unpacked(q, scale, "f32").cpu()
    bad = torch.zeros(12, dtype=torch.bool)
    bad[3] = bad[4] = bad[5] = True
    assert bool(scale.cpu()[bad].isnan().all()) and bool((q.cpu()[bad] == 0).all())
    assert bool(back[bad].isnan().all()) and not bool(back[~bad].isnan().any())
    check_packed(q[~bad.cuda()], scale[~bad.cuda()], x[~bad].double(), 0.0)
    assert bool((back[1] == 0).all()) and bool((q[6] == 127).all()) and bool((q[7] == -127).all())
    assert bool((q[2, :-1] == 0).all()) and int(q[2, -1]) == 127
    # every bit of a NaN: none of it reaches the bytes
    y = x.float()
    y.view(torch.int32)[3, width // 2] = 0x7f812345
    assert bool((rows8().packed(y.cuda())[0][3] == 0).all())


def test_ties_go_to_the_even_number():
    """A scale of exactly 1: the largest value is 127."""
    x = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 3.49, 3.51, 126.5]])
    q, scale = rows8().packed(x.cuda())
    assert float(scale[0]) == 1.0
    assert q.cpu().tolist() == [[127, 0, 2, 2, 0, -2, 3, 4, 126]]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quotients_of_the_smallest_rows(dtype):
    """Rows whose largest value is 2^-126 to 2^-95, with values in the middle of
    two bytes and next to it: x - q s is then as small as binary32's smallest
    numbers, and the bytes are still those of a division (rounded once, ties of
    rint to even)."""
    M, C = 4000, 61
    g = torch.Generator().manual_seed(11)
    largest = torch.exp2(torch.randint(-126, -95, (M, 1), generator=g).float()) * (1.0 + torch.rand((M, 1), generator=g))
    largest = largest.to(DTYPES[dtype]).float()
    scale = (largest / 127.0).clamp(min=LEAST)
    x = scale * (torch.randint(0, 127, (M, C), generator=g).float() + 0.5)
    x = (x.view(torch.int32) + torch.randint(-1, 2, (M, C), generator=g, dtype=torch.int32)).view(torch.float32)
    x = torch.minimum(x, largest) * (2.0 * torch.randint(0, 2, (M, C), generator=g) - 1.0)
    x[:, :1] = largest
    x = x.to(DTYPES[dtype])
    x[:, 1:] = torch.where(x[:, 1:].abs() > x[:, :1], x[:, :1], x[:, 1:])      # (a rounding to bf16 may pass it)
    q, got = rows8().packed(x.cuda())
    assert torch.equal(got.cpu(), scale[:, 0])
    assert torch.equal(q.cpu(), torch.round(x.float() / scale).to(torch.int8))


def test_a_second_packing_changes_nothing():
    """The values of rows in 8 bits, packed again, are the same rows (their
    largest is 127 s to a rounding)."""
    q, scale = rows8().packed(matrix(500, 300, "f32", 1).cuda())
    again, other = rows8().packed(rows8().unpacked(q, scale, "f32"))
    assert torch.equal(q, again) and float(((other - scale) / scale).abs().max()) <= 2.0 ** -22


def test_strided_rows_columns_and_slices():
    """Every second row; a column of a matrix, whose stride is a row's."""
    big = matrix(64, 200, "bf16", 3).cuda()
    q, scale = rows8().packed(big[::2])
    want, want_scale = rows8().packed(big[::2].contiguous())
    assert torch.equal(q, want) and torch.equal(scale, want_scale)
    q1, s1 = rows8().packed(big[:, 7:8])
    assert torch.equal(q1.float() * s1[:, None], torch.sign(q1.float()) * 127 * s1[:, None])
    one, s_one = rows8().packed(big[5:6])
    all_, s_all = rows8().packed(big)
    assert torch.equal(one[0], all_[5]) and torch.equal(s_one[0], s_all[5])


def test_streams_and_graphs():
    xs = [matrix(2000, 320, "f16", 10 + i).cuda() for i in range(3)]
    want = [rows8().packed(x) for x in xs]
    back = [rows8().unpacked(q, s, "f16") for q, s in want]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    q, s = rows8().packed(xs[1], stream=side)
    v = rows8().unpacked(q, s, "f16", stream=side)
    side.synchronize()
    assert torch.equal(q, want[1][0]) and torch.equal(s, want[1][1]) and torch.equal(v, back[1])
    x = xs[0].clone()
    q, s, v = torch.empty_like(want[0][0]), torch.empty_like(want[0][1]), torch.empty_like(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert rows8().pack(x, q, s) == 0 and rows8().unpack(q, s, v) == 0
    for step in range(6):
        i = step % 3
        x.copy_(xs[i])
        for t in (q, s, v):
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q, want[i][0]) and torch.equal(s, want[i][1]) and torch.equal(v, back[i]), step
        if step % 2:
            assert torch.equal(rows8().packed(xs[2 - i])[0], want[2 - i][0])


def test_no_rows():
    q, scale = rows8().packed(torch.empty((0, 40), dtype=torch.float16, device="cuda"))
    assert q.shape == (0, 40) and scale.shape == (0,)
    assert rows8().unpacked(q, scale, "bf16").shape == (0, 40)


def test_offsets_beyond_32_bits():
    """Rows 2^29 elements apart: the last one starts beyond 2^32."""
    width, ld, rows = 500, 1 << 29, 10
    store = torch.empty(ld * (rows - 1) + width, dtype=torch.int8, device="cuda")
    q = store.as_strided((rows, width), (ld, 1))
    x = matrix(rows, width, "f16", 3).cuda()
    scale = torch.empty(rows, device="cuda")
    assert rows8().pack(x, q, scale) == 0
    want, want_scale = rows8().packed(x)
    assert torch.equal(q.contiguous(), want) and torch.equal(scale, want_scale)
    v = torch.empty_like(x)
    assert rows8().unpack(q, scale, v) == 0
    assert torch.equal(v, rows8().unpacked(want, want_scale, "f16"))
    # more than 2^32 elements in all
    del store, q
    n, big = 5000, 900_000
    part = matrix(n, 4900, "bf16", 4).cuda()
    x = part.repeat(big // n, 1)
    q, scale = rows8().packed(x)
    assert torch.equal(q[-n:], q[:n]) and torch.equal(scale[-n:], scale[:n])
    check_packed(q[-n:], scale[-n:], part.double(), 0.0)
    v = rows8().unpacked(q, scale, "bf16")
    assert torch.equal(v[-n:], (q[-n:].float() * scale[-n:, None]).to(torch.bfloat16))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_rows_that_the_caches_do_not_hold(dtype):
    """300,000 x 512: written past the caches, in whole lines; the same rows in
    pieces, and in wider ones that are not, are written through them."""
    M, C = 300_000, 512
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((M, C), generator=g, device="cuda").to(DTYPES[dtype])
    q, scale = rows8().packed(x)
    v = rows8().unpacked(q, scale, dtype)
    for lo in range(0, M, 100_000):
        part = slice(lo, lo + 100_000)
        assert torch.equal(rows8().unpacked(q[part], scale[part], dtype), v[part])
    wide = torch.full((M, C + 8), 77.0, dtype=DTYPES[dtype], device="cuda")
    assert rows8().unpack(q, scale, wide[:, :C]) == 0
    assert torch.equal(wide[:, :C], v) and bool((wide[:, C:] == 77.0).all())
