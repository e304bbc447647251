"""Norm, dropout and dense products from their definitions in 64 bits on the CPU, with bounds of what 32-bit sums and
functions and one rounding to the output's type may add."""
import math

import numpy as np
import torch

from layer_reference import ROUND, TINY, rounded  # noqa: F401

U = 2.0 ** -24
ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh"]


def chain(n):
    """Additions on the way of one value into a row's sum: a thread's own values (up to 64 of them, or a 256th of a long
    row) and some levels of joining threads."""
    return 64 + n / 256 + 16


def norm(x, w, b, eps, center):
    """y, its bound before the rounding, stats and theirs.  With d the deviations from a first mean, whose own error
    makes them larger by `off`: shift and variance are sums of chain() additions, and each step after them rounds."""
    x = x.double()
    H = x.shape[1]
    w = torch.ones(H, dtype=torch.float64) if w is None else w.double()
    b = torch.zeros(H, dtype=torch.float64) if b is None else b.double()
    m = x.mean(1, keepdim=True) if center else torch.zeros(x.shape[0], 1, dtype=torch.float64)
    d = x - m
    var = (d * d).mean(1, keepdim=True)
    r = (var + eps) ** -0.5
    off = chain(H) * U * x.abs().mean(1, keepdim=True) if center else 0.0
    d0 = d.abs() + off
    e_shift = (chain(H) * U * d0.mean(1, keepdim=True) + U * m.abs()) if center else torch.zeros_like(m)
    e_d = 2 * U * d0 + chain(H) * U * d0.mean(1, keepdim=True) * center
    e_r = r * (0.5 * (chain(H) + 6) * U * (d0 * d0).mean(1, keepdim=True) / (var + eps) + 4 * U)
    y = d * r * w + b
    err = w.abs() * (e_d * (r + e_r) + d.abs() * e_r + 3 * U * d.abs() * r) + 2 * U * (y.abs() + b.abs())
    return y, err, torch.cat([m, r], 1), torch.cat([e_shift + U * m.abs(), e_r], 1)


def norm_grad(dy, x, stats, w, center, residual=None):
    """d_x, d_weight, d_bias and their bounds, for given statistics."""
    dy, x, m, r = dy.double(), x.double(), stats[:, :1].double(), stats[:, 1:].double()
    T, H = x.shape
    w = torch.ones(H, dtype=torch.float64) if w is None else w.double()
    unit, g = (x - m) * r, dy * w
    mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731
    mg = mean(g) if center else 0.0 * mean(g)
    mgu = mean(g * unit)
    dx = r * (g - mg - unit * mgu)
    err = r * U * (8 * (g.abs() + mg.abs() + (unit * mgu).abs()) + (chain(H) + 8) * (mean(g.abs()) * center + unit.abs() * mean((g * unit).abs())))
    if residual is not None:
        dx = dx + residual.double()
        err = err + U * dx.abs()
    dw, db = (dy * unit).sum(0), dy.sum(0)
    return dx, err, dw, (T + 8) * U * (dy * unit).abs().sum(0), db, (T + 8) * U * dy.abs().sum(0)


def _mixed(z):
    z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
    z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    return z ^ (z >> np.uint64(31))


def mixed(z):
    """SplitMix64's output function on an array of uint64."""
    with np.errstate(over="ignore"):
        return _mixed(np.asarray(z, dtype=np.uint64))


GAMMA = np.uint64(0x9E3779B97F4A7C15)


def kept(T, H, p, seed, step=0, first_row=0):
    """The mask bool [T, H] of rows from first_row on, and the factor."""
    with np.errstate(over="ignore"):
        key = _mixed(np.array([seed], dtype=np.uint64) + GAMMA) ^ np.array([step], dtype=np.int64).view(np.uint64)
        key = _mixed(key + GAMMA)
        W = (H + 3) // 4
        n = (np.arange(T * W, dtype=np.uint64) + np.uint64(first_row * W + 1))
        word = _mixed(key + n * GAMMA).reshape(T, W, 1)
    field = (word >> (np.arange(4, dtype=np.uint64) * np.uint64(16))).reshape(T, W * 4)[:, :H] & np.uint64(0xffff)
    least = math.floor(p * 65536 + 0.5)
    return torch.from_numpy(field.astype(np.int64) >= least), (65536 / (65536 - least) if least < 65536 else 0.0)


def dropout(x, mask, scale, residual=None):
    """out and its bound: the factor, the product and the sum each round."""
    y = torch.where(mask, x.double() * scale, 0.0)
    err = 2 * U * y.abs()
    if residual is not None:
        y = y + residual.double()
        err = err + U * y.abs()
    return y, err


def act(v, name):
    if name == "relu":
        return v.clamp(min=0)
    if name == "silu":
        return v * torch.sigmoid(v)
    if name == "gelu":
        return v * 0.5 * torch.special.erfc(-v / math.sqrt(2))
    if name == "gelu_tanh":
        return v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
    return v


def slope(v, name):
    """The activation's derivative by its formula (relu's at 0 is 0)."""
    if name == "relu":
        return (v > 0).double()
    if name == "silu":
        s = torch.sigmoid(v)
        return s * (1 + v * torch.sigmoid(-v))
    if name == "gelu":
        return 0.5 * torch.special.erfc(-v / math.sqrt(2)) + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        k = 2 * math.sqrt(2 / math.pi)
        z = k * (v + 0.044715 * v ** 3)
        s, rest = torch.sigmoid(z), torch.sigmoid(-z)
        return s * (1 + v * rest * k * (1 + 3 * 0.044715 * v * v))
    return torch.ones_like(v)


def _exponent(v, name):
    """Size of the exponential's argument: rounding it (some four roundings) is what large arguments cost."""
    k = 2 * math.sqrt(2 / math.pi)
    return {"silu": v.abs(), "gelu": v * v / 2, "gelu_tanh": k * (v + 0.044715 * v ** 3).abs()}.get(name, 0 * v)


def act_error(v, name, dv):
    """Bound of the activation's error for a value v that is off by dv: slopes are at most 1.13; evaluation costs 24 units
    (a polynomial of nine terms, an exponential, a reciprocal) and four of the exponent's."""
    if name in ("none", "relu"):
        return dv
    return 1.13 * dv + (4 * _exponent(v, name) + 24) * U * act(v, name).abs() + 1e-28


def slope_error(v, name):
    """Bound of the derivative's error at an exact v: as above, of its two terms."""
    if name in ("none", "relu"):
        return 0 * v
    if name == "silu":
        s = torch.sigmoid(v)
        size = s + v.abs() * s * torch.sigmoid(-v)
    elif name == "gelu":
        size = 0.5 * torch.special.erfc(-v / math.sqrt(2)) + v.abs() * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    else:
        k = 2 * math.sqrt(2 / math.pi)
        z = k * (v + 0.044715 * v ** 3)
        s = torch.sigmoid(z)
        size = s + v.abs() * s * torch.sigmoid(-z) * k * (1 + 3 * 0.044715 * v * v)
    return (8 * _exponent(v, name) + 32) * U * size + 1e-28


def linear(x, w, bias=None, name="none", residual=None):
    """y, its bound before the rounding, pre and its: 32-bit sums of K products in any order."""
    xd, wd = x.double(), w.double()
    z, e = xd @ wd.t(), (w.shape[1] + 2) * U * (xd.abs() @ wd.abs().t())
    if bias is not None:
        z = z + bias.double()
        e = e + U * z.abs()
    y, err = act(z, name), act_error(z, name, e)
    if residual is not None:
        y = y + residual.double()
        err = err + U * y.abs()
    return y, err, z, e


def act_grad(dy, pre, name):
    """d_pre, d_bias and their bounds."""
    dy = dy.double()
    if name == "none":
        d, e = dy, 0 * dy
    else:
        v = pre.double()
        d = dy * slope(v, name)
        e = dy.abs() * slope_error(v, name) + 3 * U * d.abs()
    return d, e, d.sum(0), e.sum(0) + (len(dy) + 4) * U * d.abs().sum(0)


def linear_grad_x(dy, w, name="none", pre=None, residual=None):
    dyd, wd = dy.double(), w.double()
    dx, e = dyd @ wd, (w.shape[0] + 2) * U * (dyd.abs() @ wd.abs())
    if name != "none":
        v = pre.double()
        e = e * (slope(v, name).abs() + slope_error(v, name)) + dx.abs() * slope_error(v, name)
        dx = dx * slope(v, name)
        e = e + 3 * U * dx.abs()
    if residual is not None:
        dx = dx + residual.double()
        e = e + U * dx.abs()
    return dx, e


def linear_grad_w(dy, x):
    dyd, xd = dy.double(), x.double()
    return dyd.t() @ xd, (len(dy) + 2) * U * (dyd.abs().t() @ xd.abs())
