"""The layer operators from their definitions in 64 bits (torch, CPU or GPU), and how far a result in its type may be off.

u(t) is half a step of a 16-bit type relative to the value (2^-11 for float16, 2^-8 for bfloat16), tiny(t) half its smallest
step; E = 2^-24 is half a step of float32, in which statistics, sums and products are held."""
import math

import torch

E = 2.0 ** -24
DT = {"f16": torch.float16, "bf16": torch.bfloat16}
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}


def u(t):
    return torch.finfo(t).eps / 2


def tiny(t):
    return 2.0 ** -25 if t == torch.float16 else 2.0 ** -134


def encode(x):
    """int8 rows and float32 scales by whole-number arithmetic: q is the whole number nearest to 127 x / amax, ties to even."""
    x = x.double()
    finite = torch.where(torch.isfinite(x), x, torch.zeros_like(x))
    amax = finite.abs().amax(dim=1, keepdim=True)
    safe = torch.where(amax > 0, amax, torch.ones_like(amax))
    low = torch.floor(127.0 * finite / safe)
    twice = 2.0 * (127.0 * finite - low * safe)            # against safe: above, up; below, down; equal, to the even one
    q = torch.where((twice > safe) | ((twice == safe) & (torch.remainder(low, 2) == 1)), low + 1, low)
    q = torch.where(torch.isinf(x), torch.sign(x) * 127.0, q)
    q = torch.where(torch.isnan(x), torch.zeros_like(q), q)
    # torch divides by a number as a product with its rounded reciprocal; a quotient of tensors in 64 bits, rounded once more, is the
    # float32 quotient
    return q.to(torch.int8), (amax / torch.full_like(amax, 127.0)).float().reshape(-1)


def value(tensor, scale=None):
    v = tensor.double()
    return v if scale is None else v * scale.double()[:, None]


def phi(z):
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))


def activate(z, act):
    if act == "relu":
        return torch.relu(z)
    if act == "gelu":
        return z * phi(z)
    if act == "silu":
        return z * torch.sigmoid(z)
    return z.clone()


def slope(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return phi(z) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1.0 - s)
    return torch.ones_like(z)


def norm(x, gamma, beta, eps, centred):
    mean = x.mean(dim=1) if centred else torch.zeros(x.shape[0], dtype=torch.float64, device=x.device)
    d = x - mean[:, None]
    rstd = 1.0 / torch.sqrt(d.square().mean(dim=1) + eps)
    y = d * rstd[:, None]
    if gamma is not None:
        y = y * gamma
    if beta is not None:
        y = y + beta
    return y, mean, rstd


def norm_backward(dy, x, gamma, mean, rstd, centred):
    h = (x - (mean[:, None] if centred else 0.0)) * rstd[:, None]
    g = dy * gamma if gamma is not None else dy
    dx = g - h * (g * h).mean(dim=1, keepdim=True)
    if centred:
        dx = dx - g.mean(dim=1, keepdim=True)
    return dx * rstd[:, None], (dy * h).sum(dim=0), dy.sum(dim=0)


# ---- how far off ---------------------------------------------------------------------------------------------------
def norm_bound(x, gamma, beta, y, rstd, t, centred):
    """A sum of n float32 terms by lanes and a tree over them has at most 32 + 16 roundings in a row, so the mean is off by 48 E mean|x|;
    x - mean adds one rounding; the root of the mean square is off by half of (two for the squares, 48 for the sum, and what the differences are off) and four more
    for the division and the root; three products and a sum follow."""
    ax = x.abs()
    off = E * (2.0 * ax + 64.0 * ax.mean(dim=1, keepdim=True)) if centred else E * ax
    g = gamma.abs() if gamma is not None else torch.ones(x.shape[1], dtype=torch.float64, device=x.device)
    rel = 60.0 * E + (off.square().mean(dim=1, keepdim=True).sqrt()) * rstd[:, None]
    h = (y - (beta if beta is not None else 0.0)).abs()
    err = off * rstd[:, None] * g + rel * h + 4.0 * E * (h + y.abs())
    return err + u(t) * (y.abs() + err) + tiny(t)


def norm_backward_bounds(dy, x, gamma, mean, rstd, dx, t, centred):
    """h has three roundings and what x - mean cancels; g h, their sums (48 in a row, n of them shared) and the last three operations
    follow.  A column sum over the rows has at most rows + 64 roundings in a row."""
    n = x.shape[1]
    mu = mean[:, None] if centred else torch.zeros_like(rstd)[:, None]
    h = ((x - mu) * rstd[:, None]).abs()
    dh = 3.0 * E * h + 2.0 * E * (x.abs() + mu.abs()) * rstd[:, None]
    g = (dy * gamma).abs() if gamma is not None else dy.abs()
    mg = g.mean(dim=1, keepdim=True)
    mgh = (g * h).mean(dim=1, keepdim=True)
    e_mgh = 56.0 * E * mgh + (g * dh).mean(dim=1, keepdim=True)
    err = rstd[:, None] * (dh * mgh + h * e_mgh + 56.0 * E * mg + 6.0 * E * (g + mg + h * mgh))
    rows = x.shape[0]
    dgamma = ((rows + 64) * E * (dy.abs() * h) + dy.abs() * dh).sum(dim=0)
    dbeta = (rows + 64) * E * dy.abs().sum(dim=0)
    return err + u(t) * (dx.abs() + err) + tiny(t), dgamma, dbeta


def product_error(pabs, terms):
    """a float32 sum of `terms` exact products whose magnitudes add up to pabs, in any order"""
    return (terms + 8) * E * pabs


def activation_error(z, act):
    """the exponential's argument is rounded (|z| log2 e, z^2 / 2), the rest is a few roundings of values of z's size; the tail's published error is 7.5e-8"""
    if act in ("gelu", "silu"):
        return z.abs() * (2e-7 + 8.0 * E) + 2.0 * E * (1.0 + z.abs())
    return torch.zeros_like(z)


def slope_error(z, act):
    """the same without the factor z in front and once with it: z times the bell curve or s (1 - s), both under 0.4 and falling faster than z grows"""
    return torch.full_like(z, 8e-7) if act in ("gelu", "silu") else torch.zeros_like(z)


def worst(got, want, bound):
    """largest error in units of its bound; NaN and infinities have to be alike"""
    got = got.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    ratio = torch.where(same, torch.zeros_like(want), (got - want).abs() / bound)
    ratio = torch.where(torch.isnan(ratio), torch.full_like(ratio, float("inf")), ratio)
    return ratio.max().item() if ratio.numel() else 0.0
