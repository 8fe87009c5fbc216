"""Plain 64-bit restatements of the head operators, for the tests."""
import math

import torch

U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}      # half a unit in the last place, relative
TINY = {"f32": 0.0, "f16": 2.0 ** -25, "bf16": 0.0}                # half the spacing of the subnormals
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ACTS = ("none", "relu", "silu", "gelu")
E32 = 2.0 ** -24


def activation(act, u):
    if act == "relu":
        return u.clamp(min=0.0)
    if act == "silu":
        return u * torch.special.expit(u)
    if act == "gelu":
        return u * 0.5 * torch.special.erfc(-u / math.sqrt(2.0))
    return u.clone()


def activation_grad(act, u):
    if act == "relu":
        return (u > 0).double()
    if act == "silu":
        s = torch.special.expit(u)
        return s * (1.0 + u * (1.0 - s))
    if act == "gelu":
        return 0.5 * torch.special.erfc(-u / math.sqrt(2.0)) + u * torch.exp(-0.5 * u * u) / math.sqrt(2 * math.pi)
    return torch.ones_like(u)


def norm_sample(x, gamma, beta, groups, act, eps):
    """One sample's (P, C) pixels in 64 bits: y, mean [G], rstd [G]."""
    P, C = x.shape
    v = x.reshape(P, groups, C // groups)
    mean = v.mean((0, 2))
    d = v - mean[None, :, None]
    rstd = 1.0 / torch.sqrt((d * d).mean((0, 2)) + eps)
    u = (d * rstd[None, :, None]).reshape(P, C) * gamma + beta
    return activation(act, u), mean, rstd


def norm(x, gamma, beta, groups, act, eps, sizes):
    """(B, P, C) in 64 bits: y (0 from each sample's size on), stats [B][G][2]."""
    y = torch.zeros_like(x)
    stats = torch.zeros((x.shape[0], groups, 2), dtype=torch.float64)
    for b, n in enumerate(sizes):
        if n == 0:
            stats[b, :, 1] = 1.0 / math.sqrt(eps)
            continue
        y[b, :n], stats[b, :, 0], stats[b, :, 1] = norm_sample(x[b, :n], gamma, beta, groups, act, eps)
    return y, stats


def norm_grad(x, dy, gamma, beta, groups, act, eps, sizes):
    """The gradient's formulas in 64 bits: dx, dgamma, dbeta, and the sums of
    the absolute terms of the last two."""
    B, P, C = x.shape
    dx = torch.zeros_like(x)
    dgamma, dbeta, agamma, abeta = (torch.zeros(C, dtype=torch.float64) for _ in range(4))
    for b, n in enumerate(sizes):
        if n == 0:
            continue
        _, mean, rstd = norm_sample(x[b, :n], gamma, beta, groups, act, eps)
        cpg = C // groups
        m, r = mean.repeat_interleave(cpg), rstd.repeat_interleave(cpg)
        xh = (x[b, :n] - m) * r
        du = dy[b, :n] * activation_grad(act, xh * gamma + beta)
        t = (du * gamma).reshape(n, groups, cpg)
        a = t.sum((0, 2)) / (n * cpg)
        q = (t * xh.reshape(n, groups, cpg)).sum((0, 2)) / (n * cpg)
        dx[b, :n] = r * (du * gamma - a.repeat_interleave(cpg) - xh * q.repeat_interleave(cpg))
        dgamma += (du * xh).sum(0)
        dbeta += du.sum(0)
        agamma += (du * xh).abs().sum(0)
        abeta += du.abs().sum(0)
    return dx, dgamma, dbeta, agamma, abeta


def inside(got, want, bound, what):
    """|got - want| <= bound everywhere, NaNs in the same places."""
    got, want = got.detach().cpu().double(), want.double()
    assert got.shape == want.shape, what
    assert torch.equal(got.isnan(), want.isnan()), f"{what}: NaNs differ"
    ok = ~want.isnan()
    far = ((got - want).abs() - bound)[ok] if torch.is_tensor(bound) else ((got - want).abs() - bound)[ok]
    far = far[~far.isnan()]          # equal infinities
    assert far.numel() == 0 or float(far.max()) <= 0.0, f"{what}: {float(far.max()):.3g} beyond its bound"
