"""Plain restatements of the operators on rows in 8 bits, and the helpers of
their tests."""
import torch

from tests.headref import DTYPES, E32

LEAST = 2.0 ** -126


def matrix(rows, width, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn((rows, width), generator=g)).to(DTYPES[dtype])


def byte_rows(rows, width, seed, scale=1.0, whole_range=False):
    """Rows in 8 bits as they are packed from normal values, each of a size of
    its own: (int8, float32 scales)."""
    g = torch.Generator().manual_seed(seed)
    if whole_range:
        return (torch.randint(-128, 128, (rows, width), generator=g, dtype=torch.int8),
                scale * (0.5 + torch.rand(rows, generator=g)))
    x = scale * torch.randn((rows, width), generator=g) * torch.exp(0.5 * torch.randn((rows, 1), generator=g))
    s = (x.abs().amax(1) / 127.0).clamp(min=LEAST)
    return torch.round(x / s[:, None]).to(torch.int8), s


def values(q, scale):
    """What rows in 8 bits stand for, in 64 bits."""
    return q.double() * scale.double()[:, None]


def padded(m, pad, lead=0):
    """On the GPU, each row inside a wider one of values that are not its own."""
    rows, width = m.shape
    if m.dtype is torch.int8:
        full = torch.full((rows, width + pad + lead), 93, dtype=torch.int8, device="cuda")
    else:
        full = torch.full((rows, width + pad + lead), float("nan"), dtype=m.dtype, device="cuda")
    full[:, lead:lead + width] = m.cuda()
    return full[:, lead:lead + width]


def target(rows, width, pad, dtype, lead=0):
    """A buffer of 77s and the view of its rows."""
    t = torch.int8 if dtype == "i8" else DTYPES[dtype]
    full = torch.full((rows + 1, width + pad + lead), 77, dtype=t, device="cuda")
    return full, full[:rows, lead:lead + width]


def untouched(full, view):
    """Whether everything but the view's rows still holds 77."""
    rest = full.clone()
    lead = view.storage_offset() - full.storage_offset()
    rest[:view.shape[0], lead:lead + view.shape[1]] = 77
    return bool((rest == 77).all())


def check_packed(q, scale, y, rel):
    """Rows in 8 bits against the 64-bit values that were packed, which the
    kernel has to a relative error of `rel`: the scale is m / 127 to that and a
    rounding, and q the nearest whole number to y / s, where an error of y of
    rel, one of 1/s and the product's of 2 x 2^-24, and 127 of them, may choose
    the other one of two."""
    q, scale, y = q.cpu(), scale.cpu().double(), y.cpu().double()
    want = (y.abs().amax(1) / 127.0).clamp(min=LEAST)
    assert bool(((scale - want).abs() <= (rel + 2 * E32) * want).all())
    off = (q.double() - y / scale[:, None]).abs().max() if q.numel() else 0.0
    assert float(off) <= 0.5 + 127.5 * (rel + 3 * E32), float(off)
    assert q.numel() == 0 or int(q.min()) >= -127
