"""The work that the head operators are measured on: group norm with an
activation over channels-last maps, and the matrix product with bias,
activation and residual in its epilogue, each with its gradient.

``run`` computes a case either in its plain form (elementary torch operations
in 32 bits, rounded once) or, with ``own`` set, through the package's public
binding; ``exact`` restates the definitions in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

EPS = 1e-5
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def _norm(name, op, samples, pixels, channels, groups, dtype, act, valid=False, pad=0):
    """A group norm case; ``valid``: each sample has its own number of pixels
    (the first one none), ``pad``: elements between the rows of two pixels."""
    case = {"op": op, "B": samples, "P": pixels, "C": channels, "G": groups, "dtype": dtype, "act": act,
            "valid": valid, "pad": pad}
    return {"name": name, **case} if name else case


def _linear(name, op, rows, k, n, dtype, act, residual=False, save=False, pad=0):
    """A matrix product case; ``save``: the forward also stores the value
    before the activation, as the gradient needs it."""
    case = {"op": op, "M": rows, "K": k, "N": n, "dtype": dtype, "act": act, "residual": residual, "save": save,
            "pad": pad}
    return {"name": name, **case} if name else case


def listed():
    return [
        # a 64x64 crop on its way through a small head: a launch-latency case
        _norm("norm_crop_64", "norm", 1, 64 * 64, 64, 8, "f32", "silu"),
        # the feature map of one 640x640 frame, before the projection to its embedding
        _norm("norm_frame_640", "norm", 1, 640 * 640, 256, 32, "f16", "silu"),
        # a served batch of images of different sizes, as rows of backbone features
        _norm("norm_ragged_batch", "norm", 16, 1024, 1024, 32, "bf16", "gelu", valid=True),
        # a training step on four 256x256 maps
        _norm("norm_grad_256", "norm_grad", 4, 256 * 256, 64, 16, "f16", "silu"),
        # a training step on a street scene
        _norm("norm_grad_street", "norm_grad", 1, 1024 * 2048, 64, 8, "bf16", "silu"),
        # odd sizes, few channels to a group, rows inside a wider buffer, single precision
        _norm("norm_grad_odd", "norm_grad", 1, 479 * 641, 100, 25, "f32", "gelu", pad=12),
        # one row, as a served query asks for: bound by the weights
        _linear("linear_row", "linear", 1, 1024, 1024, "f16", "silu", residual=True),
        # a backbone block's wide product over the 44x44 patches of an image, kept for the gradient
        _linear("linear_wide", "linear", 44 * 44, 1024, 4096, "bf16", "gelu", save=True),
        # the projection of a 640x640 feature map to the embedding that the decoder reads
        _linear("linear_embed_640", "linear", 640 * 640, 256, 64, "f16", "none"),
        # odd sizes in single precision
        _linear("linear_odd", "linear", 71 * 73, 100, 65, "f32", "silu", residual=True, pad=3),
        # the projection's gradient, a hidden layer's with its activation
        _linear("linear_grad_640", "linear_grad", 640 * 640, 256, 64, "f16", "silu"),
        # the wide product's gradient over a batch of four images
        _linear("linear_grad_wide", "linear_grad", 4 * 44 * 44, 1024, 4096, "bf16", "gelu"),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _common(size):
    """3072 is no size of this package's workloads."""
    return 3136 if size == 3072 else size


def draw(rng: random.Random):
    """One more case of the same ranges."""
    op = rng.choice(["norm", "norm_grad", "linear", "linear_grad"])
    dtype = rng.choice(["f16", "bf16", "f16", "bf16", "f32"])
    act = rng.choice(["none", "relu", "silu", "gelu"])
    if op.startswith("norm"):
        per = rng.choice([1, 2, 3, 4, 5, 8, 8, 16, 24, 32])
        groups = rng.choice([1, 2, 4, 7, 8, 16, 25, 32])
        while per * groups > 1024 or per * groups < 8:
            per, groups = rng.choice([2, 4, 8, 16]), rng.choice([4, 8, 16, 32])
        elements = _log_uniform(rng, 1 << 17, 1 << 26 if dtype == "f32" else 1 << 27)
        samples = rng.choice([1, 1, 1, 2, 4, rng.randint(1, 16)])
        pixels = _common(max(1, min(2048 * 1024, elements // (samples * per * groups))))
        return _norm("", op, samples, pixels, per * groups, groups, dtype, act, rng.random() < 0.25,
                     rng.choice([0, 0, 0, 8, 16, rng.randint(1, 31)]))
    k, n = _log_uniform(rng, 16, 4096), _log_uniform(rng, 16, 4096)
    if rng.random() < 0.7:
        k, n = (k + 7) // 8 * 8, (n + 7) // 8 * 8
    if rng.random() < 0.4:
        k, n = (k + 63) // 64 * 64, (n + 63) // 64 * 64
    k, n = _common(k), _common(n)
    flops = (3 << 32) if dtype == "f32" else (1 << 34)
    most = int(min(640 * 640, flops // (k * n), (1 << 26) // max(k, n)))
    rows = _common(_log_uniform(rng, 1, max(2, most)))
    return _linear("", op, rows, k, n, dtype, act, op == "linear" and rng.random() < 0.4,
                   op == "linear" and rng.random() < 0.3, rng.choice([0, 0, 0, 8, 16, rng.randint(1, 31)]))


# -- inputs -----------------------------------------------------------------------

def _rows(gen, shape, pad, dtype, scale=1.0, shift=0.0):
    """Normal values, each last-axis row followed by ``pad`` elements that do
    not belong to it."""
    full = scale * torch.randn(shape[:-1] + (shape[-1] + pad,), generator=gen, device="cuda")
    full[..., :shape[-1]] += shift
    return full.to(dtype)[..., :shape[-1]]


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _lengths(case, seed):
    """Pixels of each sample: the first sample has none where there are others."""
    if not case["valid"]:
        return None
    rng = random.Random(seed * 7919 + case["P"])
    sizes = [rng.randint(max(1, case["P"] // 4), case["P"]) for _ in range(case["B"])]
    if case["B"] > 1:
        sizes[0] = 0
    return sizes


def _inputs(case, seed):
    gen, dtype = _generator(seed), DTYPES[case["dtype"]]
    if case["op"].startswith("norm"):
        B, P, C = case["B"], case["P"], case["C"]
        shift = 0.5 * torch.randn(C, generator=gen, device="cuda")      # channels have means of their own
        s = {"x": _rows(gen, (B, P, C), case["pad"], dtype, 1.5, shift),
             "gamma": 1.0 + 0.2 * torch.randn(C, generator=gen, device="cuda"),
             "beta": 0.3 * torch.randn(C, generator=gen, device="cuda"), "valid": None}
        sizes = _lengths(case, seed)
        if case["op"] == "norm_grad":
            s["dy"] = _rows(gen, (B, P, C), case["pad"], dtype, 0.1)
        if sizes is not None:
            s["valid"] = torch.tensor(sizes, dtype=torch.int32, device="cuda")
            behind = (torch.arange(P, device="cuda")[None, :] >= s["valid"][:, None])[:, :, None]
            s["x"].masked_fill_(behind, float("nan"))       # what lies behind a sample's pixels was never written
            if "dy" in s:
                s["dy"].masked_fill_(behind, float("nan"))
        if case["op"] == "norm_grad":
            s["stats"] = _statistics(s["x"], s["valid"], case["G"])
        return s
    M, K, N = case["M"], case["K"], case["N"]
    s = {"x": _rows(gen, (M, K), case["pad"], dtype), "w": _rows(gen, (N, K), 0, dtype, K ** -0.5)}
    if case["op"] == "linear":
        s["bias"] = 0.2 * torch.randn(N, generator=gen, device="cuda")
        s["residual"] = _rows(gen, (M, N), case["pad"], dtype) if case["residual"] else None
    else:
        s["dy"] = _rows(gen, (M, N), case["pad"], dtype, 0.1)
        s["z"] = _rows(gen, (M, N), case["pad"], dtype) if case["act"] != "none" else None
    return s


def _statistics(x, valid, groups):
    """Mean and 1/sqrt(var + eps) of every sample's groups, as a forward pass leaves them."""
    B, P, C = x.shape
    sizes = torch.full((B,), P, device="cuda") if valid is None else valid
    kept = (torch.arange(P, device="cuda")[None, :] < sizes[:, None])[:, :, None, None]
    n = (sizes.double() * (C // groups)).clamp(min=1.0)[:, None]
    v = x.float().reshape(B, P, groups, -1)
    mean = (torch.where(kept, v, 0.0).sum((1, 3), dtype=torch.float64) / n).float()
    square = torch.where(kept, v - mean[:, None, :, None], 0.0).square().sum((1, 3), dtype=torch.float64)
    return torch.stack((mean, torch.rsqrt(square / n + EPS).float()), -1)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:     # the handle and the buffers that a program keeps
        from paper_2609_16874_amd import head
        dtype = DTYPES[case["dtype"]]
        if case["op"].startswith("norm"):
            shape = (case["B"], case["P"], case["C"])
            s["handle"] = head.GroupNorm(case["B"], case["P"], case["C"], case["G"], case["dtype"], case["act"], EPS)
            s["out"] = torch.empty(shape, dtype=dtype, device="cuda")
            if case["op"] == "norm":
                s["stats"] = torch.empty((case["B"], case["G"], 2), dtype=torch.float32, device="cuda")
            else:
                s["dgamma"] = torch.empty(case["C"], dtype=torch.float32, device="cuda")
                s["dbeta"] = torch.empty(case["C"], dtype=torch.float32, device="cuda")
        else:
            M, K, N = case["M"], case["K"], case["N"]
            s["handle"] = head.Linear(M, K, N, case["dtype"], case["act"])
            if case["op"] == "linear":
                s["out"] = torch.empty((M, N), dtype=dtype, device="cuda")
                s["keep"] = torch.empty((M, N), dtype=dtype, device="cuda") if case["save"] else None
            else:
                s["dx"] = torch.empty((M, K), dtype=dtype, device="cuda")
                s["dw"] = torch.empty((N, K), dtype=dtype, device="cuda")
                s["dbias"] = torch.empty(N, dtype=torch.float32, device="cuda")
    return s


# -- one pass ---------------------------------------------------------------------

def _act(act, u):
    if act == "relu":
        return u.clamp(min=0.0)
    if act == "silu":
        return u / (1.0 + torch.exp(-u))
    if act == "gelu":
        return 0.5 * u * (1.0 + torch.erf(u * math.sqrt(0.5)))
    return u


def _act_grad(act, u):
    if act == "relu":
        return (u > 0).to(u.dtype)
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-u))
        return s * (1.0 + u * (1.0 - s))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(u * math.sqrt(0.5))) + u * torch.exp(-0.5 * u * u) / math.sqrt(2.0 * math.pi)
    return torch.ones_like(u)


def _plain_norm(s, case):
    B, P, C, G = case["B"], case["P"], case["C"], case["G"]
    x, keep = s["x"].float(), None
    if s["valid"] is not None:
        keep = torch.arange(P, device="cuda")[None, :] < s["valid"][:, None]
        x = torch.where(keep[:, :, None], x, torch.zeros((), device="cuda"))
        n = (s["valid"].float() * (C // G)).clamp(min=1.0)[:, None]
    else:
        n = torch.full((B, 1), float(P * (C // G)), device="cuda")
    xg = x.reshape(B, P, G, C // G)
    if case["op"] == "norm":
        mean = xg.sum((1, 3)) / n
        d = xg - mean[:, None, :, None]
        if keep is not None:
            d = torch.where(keep[:, :, None, None], d, torch.zeros((), device="cuda"))
        rstd = 1.0 / torch.sqrt((d * d).sum((1, 3)) / n + EPS)
        u = (d * rstd[:, None, :, None]).reshape(B, P, C) * s["gamma"] + s["beta"]
        y = _act(case["act"], u)
        if keep is not None:
            y = torch.where(keep[:, :, None], y, torch.zeros((), device="cuda"))
        return {"y": y.to(s["x"].dtype), "stats": torch.stack((mean, rstd), -1)}
    mean, rstd = s["stats"][..., 0], s["stats"][..., 1]
    xh = ((xg - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(B, P, C)
    du = s["dy"].float() * _act_grad(case["act"], xh * s["gamma"] + s["beta"])
    if keep is not None:
        du = torch.where(keep[:, :, None], du, torch.zeros((), device="cuda"))
    by_sample, with_x = du.sum(1), (du * xh).sum(1)                     # [B][C]
    a = (by_sample * s["gamma"]).reshape(B, G, -1).sum(2) / n
    q = (with_x * s["gamma"]).reshape(B, G, -1).sum(2) / n
    dx = (du * s["gamma"]).reshape(B, P, G, -1) - a[:, None, :, None] - xh.reshape(B, P, G, -1) * q[:, None, :, None]
    dx = (dx * rstd[:, None, :, None]).reshape(B, P, C)
    if keep is not None:
        dx = torch.where(keep[:, :, None], dx, torch.zeros((), device="cuda"))
    return {"dx": dx.to(s["x"].dtype), "dgamma": with_x.sum(0), "dbeta": by_sample.sum(0)}


def _plain_linear(s, case):
    dtype = s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    if case["op"] == "linear":
        z = x @ w.t() + s["bias"]
        y = _act(case["act"], z)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        out = {"y": y.to(dtype)}
        if case["save"]:
            out["z"] = z.to(dtype)
        return out
    dz = s["dy"].float()
    if s["z"] is not None:
        dz = dz * _act_grad(case["act"], s["z"].float())
    return {"dx": (dz @ w).to(dtype), "dw": (dz.t() @ x).to(dtype), "dbias": dz.sum(0)}


def _checked(status):
    if status != 0:
        raise RuntimeError(f"status {status}")


def run(s):
    case = s["case"]
    norm = case["op"].startswith("norm")
    if not own:
        return _plain_norm(s, case) if norm else _plain_linear(s, case)
    h = s["handle"]
    if case["op"] == "norm":
        _checked(h.forward(s["x"], s["gamma"], s["beta"], s["out"], stats=s["stats"], valid=s["valid"]))
        return {"y": s["out"], "stats": s["stats"]}
    if case["op"] == "norm_grad":
        _checked(h.backward(s["x"], s["dy"], s["gamma"], s["beta"], s["stats"], s["out"], s["dgamma"], s["dbeta"],
                            valid=s["valid"]))
        return {"dx": s["out"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if case["op"] == "linear":
        _checked(h.forward(s["x"], s["w"], s["bias"], s["out"], residual=s["residual"], preact=s["keep"]))
        return {"y": s["out"], "z": s["keep"]} if case["save"] else {"y": s["out"]}
    _checked(h.backward(s["x"], s["w"], s["dy"], s["z"], s["dx"], s["dw"], s["dbias"]))
    return {"dx": s["dx"], "dw": s["dw"], "dbias": s["dbias"]}


# -- the same in 64 bits ----------------------------------------------------------

def _activation64(act, u):
    if act == "relu":
        return u.clamp(min=0.0)
    if act == "silu":
        return u * torch.special.expit(u)
    if act == "gelu":
        return u * 0.5 * torch.special.erfc(-u / math.sqrt(2.0))
    return u.clone()


def _norm64(x, gamma, beta, groups, act):
    """One sample's (P, C) pixels."""
    by_group = x.reshape(x.shape[0], groups, -1)
    mean = by_group.mean((0, 2), keepdim=True)
    var = (by_group - mean).pow(2).mean((0, 2), keepdim=True)
    rstd = (var + EPS).pow(-0.5)
    u = ((by_group - mean) * rstd).reshape(x.shape)
    return _activation64(act, u * gamma + beta), torch.cat((mean.reshape(-1, 1), rstd.reshape(-1, 1)), 1)


def _exact_norm(case, seed):
    s = _inputs(case, seed)
    sizes = [case["P"]] * case["B"] if s["valid"] is None else s["valid"].tolist()
    gamma, beta = s["gamma"].double(), s["beta"].double()
    grad = case["op"] == "norm_grad"
    maps = torch.zeros((case["B"], case["P"], case["C"]), dtype=torch.float64, device="cuda")
    stats, gammas, betas = [], torch.zeros_like(gamma), torch.zeros_like(beta)
    for b, size in enumerate(sizes):
        if size == 0:
            stats.append(torch.tensor([[0.0, EPS ** -0.5]] * case["G"], dtype=torch.float64, device="cuda"))
            continue
        x = s["x"][b, :size].double()
        if grad:        # by differentiating the definition
            leaves = [v.detach().clone().requires_grad_(True) for v in (x, gamma, beta)]
            y, _ = _norm64(*leaves, case["G"], case["act"])
            dx, dgamma, dbeta = torch.autograd.grad(y, leaves, s["dy"][b, :size].double())
            maps[b, :size] = dx
            gammas += dgamma
            betas += dbeta
        else:
            maps[b, :size], st = _norm64(x, gamma, beta, case["G"], case["act"])
            stats.append(st)
    if grad:
        return {"dx": maps, "dgamma": gammas, "dbeta": betas}
    return {"y": maps, "stats": torch.stack(stats)}


def _exact_linear(case, seed):
    s = _inputs(case, seed)
    x, w = s["x"].double(), s["w"].double()
    if case["op"] == "linear":
        z = torch.addmm(s["bias"].double(), x, w.t())
        y = _activation64(case["act"], z)
        if s["residual"] is not None:
            y += s["residual"].double()
        return {"y": y, "z": z} if case["save"] else {"y": y}
    dz = s["dy"].double()
    if s["z"] is not None:
        z = s["z"].double().requires_grad_(True)
        (dz,) = torch.autograd.grad(_activation64(case["act"], z), z, dz)
    return {"dx": torch.mm(dz, w), "dw": torch.mm(dz.t(), x), "dbias": dz.sum(0)}


def exact(case, seed):
    with torch.enable_grad():
        return _exact_norm(case, seed) if case["op"].startswith("norm") else _exact_linear(case, seed)


def work(case):
    size = SIZE[case["dtype"]]
    if case["op"].startswith("norm"):
        n = case["B"] * case["P"] * case["C"]
        maps = 2 if case["op"] == "norm" else 3
        vectors = 4 * ((2 if case["op"] == "norm" else 4) * case["C"] + 2 * case["B"] * case["G"])
        return {"bytes": maps * n * size + vectors, "flops": (12 if case["op"] == "norm" else 24) * n}
    M, K, N = case["M"], case["K"], case["N"]
    if case["op"] == "linear":
        maps = 1 + int(case["residual"]) + int(case["save"])
        return {"bytes": (M * K + N * K + maps * M * N) * size + 4 * N, "flops": 2 * M * N * K}
    maps = 1 + int(case["act"] != "none")
    return {"bytes": (2 * M * K + 2 * N * K + maps * M * N) * size + 4 * N, "flops": 4 * M * N * K}
