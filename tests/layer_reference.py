"""The layer operators' definitions in 64 bits, on the CPU, for the tests."""
import math

import torch

BLOCK = 32
LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
#: Largest relative error of one rounding to the type, and its smallest step's half (fp16's subnormals).
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def route_scores(x, score):
    x = x.double()
    if score == "sigmoid":
        return torch.sigmoid(x)
    top = x.amax(1, keepdim=True)
    p = torch.where(x == -math.inf, torch.zeros_like(x), torch.exp(x - torch.where(top == -math.inf, 0.0, top)))
    return p / p.sum(1, keepdim=True).clamp(min=1e-300)


def route(x, k, score="softmax", bias=None, n_groups=1, top_groups=1, group_top=1, renorm=True, scale=1.0):
    """ids, weights and, for every row, the smallest difference between unequal keys that the choice compared."""
    p = route_scores(x, score)
    T, E = p.shape
    key = p if bias is None else p + bias.double()
    if bias is None and n_groups == 1:
        key = x.double()
    key = torch.where(x.double() == -math.inf, -math.inf, key)
    margin = torch.full((T,), math.inf, dtype=torch.float64)

    def closest(s):
        d = s[:, :-1] - s[:, 1:]
        d = torch.where((d > 0) & torch.isfinite(d), d, math.inf)
        return d.amin(1) if d.shape[1] else margin

    if n_groups > 1:
        per = key.view(T, n_groups, -1)
        best = per.sort(2, descending=True).values[:, :, :group_top]
        value = torch.where(best == -math.inf, 0.0, best).sum(2)
        value = torch.where(best[:, :, 0] == -math.inf, -math.inf, value)
        order = torch.sort(value, dim=1, descending=True, stable=True)
        margin = torch.minimum(margin, closest(order.values))
        kept = torch.zeros((T, n_groups), dtype=torch.bool).scatter_(1, order.indices[:, :top_groups], True)
        key = torch.where(kept[:, :, None], per, -math.inf).view(T, E)
    order = torch.sort(key, dim=1, descending=True, stable=True)
    margin = torch.minimum(margin, closest(order.values[:, :k + 1]))
    ids = order.indices[:, :k]
    chosen = torch.where(key.gather(1, ids) == -math.inf, 0.0, p.gather(1, ids))
    if renorm:
        total = chosen.sum(1, keepdim=True)
        weights = torch.where(total > 0, scale * chosen / total.clamp(min=1e-300), 0.0)
    else:
        weights = scale * chosen
    return ids, weights, margin


def route_weights(x, ids, score, renorm, scale):
    """The weights of given choices, differentiable by x."""
    p = torch.softmax(x, 1) if score == "softmax" else torch.sigmoid(x)
    chosen = p.gather(1, ids)
    return scale * (chosen / chosen.sum(1, keepdim=True) if renorm else chosen)


def silu(g):
    return g * torch.sigmoid(g)


def product(x, w, cuts, gated=False, out=None):
    """y, and a bound of the error of 32-bit sums in any order, before the last rounding."""
    n = w.shape[1]
    width = n // 2 if gated else n
    y = torch.zeros((x.shape[0], width), dtype=torch.float64)
    err = torch.zeros_like(y)
    unit = (w.shape[2] + 2) * 2.0 ** -24
    for e in range(w.shape[0]):
        a, b = cuts[e], cuts[e + 1]
        xe, we = x[a:b].double(), w[e].double()
        z, size = xe @ we.t(), unit * (xe.abs() @ we.abs().t())
        if gated:
            g, u, dg, du = z[:, :width], z[:, width:], size[:, :width], size[:, width:]
            # |silu'| <= 1.1; exp, divide and multiply add a few units of the last place
            err[a:b] = 1.1 * dg * (u.abs() + du) + silu(g).abs() * du + 2.0 ** -21 * (silu(g) * u).abs()
            z = silu(g) * u
        else:
            err[a:b] = size
        y[a:b] = z
    return y, err


def rounded(err, y, dtype):
    """The whole error bound of y after one rounding to `dtype`."""
    return err + ROUND[dtype] * (y.abs() + err) * 1.01 + TINY[dtype]


def mx_power(x):
    """Exponent (no bias) of every block of x [R, K]."""
    top = x.double().view(x.shape[0], -1, BLOCK).abs().amax(2)
    e = torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - 2
    return torch.where(top > 0, e.clamp(min=-127), torch.full_like(e, -127.0))


def mx_values(x):
    """x [R, K] after quantisation: the nearest level by comparing all of them, ties to the even code."""
    unit = torch.exp2(mx_power(x))[:, :, None]
    v = x.double().view(x.shape[0], -1, BLOCK) / unit
    mag = v.abs().clamp(max=6.0)
    d = (mag[..., None] - LEVELS).abs()
    order = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7])   # even codes first: argmin takes the first of two equal distances
    code = order[d[..., order].argmin(-1)]
    return (torch.copysign(LEVELS[code], v) * unit).reshape(x.shape)


def mx_decode(q, k):
    """The values of packed rows q [R, bytes]."""
    low, high = q[:, :k // 2] % 16, q[:, :k // 2] // 16
    code = torch.stack([low, high], 2).flatten(1).long()
    power = q[:, k // 2:k // 2 + k // BLOCK].double()
    v = torch.where(code >= 8, -LEVELS[code % 8], LEVELS[code % 8])
    scale = torch.where(power == 255, math.nan, torch.exp2(power - 127))
    return (v.view(q.shape[0], -1, BLOCK) * scale[:, :, None]).flatten(1)
