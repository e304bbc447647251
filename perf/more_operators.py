"""The dense operators of a block around a mixture-of-experts layer, as measurable cases.

Tokens are normalised (``layer_norm``), the router's logits and a shared expert are dense products with bias, activation
and residual in their epilogue (``linear``, with ``linear_act_grad``, ``linear_grad_x`` and ``linear_grad_w``), and the
layer's output meets the residual stream through dropout whose mask is made from a counter in both directions
(``dropout``).  Hidden sizes and expert counts are those of the library's named workloads.  Where ``own`` is false a pass
is written in elementary torch operations in 32 bits, rounded once at the end.
"""
import math
import types

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")
GAMMA, MIX1, MIX2 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB   # SplitMix64


def listed():
    return [
        # one decode step's tokens before the layer, root mean square only: the smallest call
        dict(name="norm-decode", kind="norm", tokens=96, hidden=4096, center=False, affine="w", params="bf16", dtype="bf16"),
        # a prefill chunk at the widest hidden size, mean and variance
        dict(name="norm-prefill", kind="norm", tokens=16384, hidden=7168, center=True, affine="wb", params="bf16",
             dtype="bf16"),
        # a training step: gradients of tokens, weight and bias, the residual branch's gradient added
        dict(name="norm-grad", kind="norm_grad", tokens=8192, hidden=4096, center=True, affine="wb", params="f32",
             residual=True, dtype="bf16"),
        # rows of an odd length, 32 bits, no vectors that are aligned in every row
        dict(name="norm-grad-odd", kind="norm_grad", tokens=4095, hidden=2047, center=True, affine="wb", params="f32",
             residual=False, dtype="f32"),
        # a training step's layer output dropped and added to the residual stream
        dict(name="dropout-residual", kind="dropout", tokens=8192, hidden=7168, p=0.1, residual=True, dtype="bf16"),
        # its gradient for a ragged batch: the same mask once more
        dict(name="dropout-grad", kind="dropout", tokens=4093, hidden=2048, p=0.25, residual=False, dtype="bf16"),
        # the router's logits of one decode step, in 32 bits
        dict(name="router-decode", kind="linear", rows=96, hidden=7168, out=256, bias=True, act="none", residual=False,
             pre=False, out_dtype="f32", dtype="bf16"),
        # the router's logits of a prefill chunk
        dict(name="router-prefill", kind="linear", rows=16384, hidden=4096, out=256, bias=False, act="none",
             residual=False, pre=False, out_dtype="f32", dtype="bf16"),
        # one decode step of a shared expert: bound by the weights' bytes
        dict(name="linear-decode", kind="linear", rows=61, hidden=4096, out=4096, bias=True, act="silu", residual=True,
             pre=False, out_dtype="bf16", dtype="bf16"),
        # a training step's shared expert, values before the activation kept for the gradient: the largest product
        dict(name="linear-train", kind="linear", rows=16381, hidden=4096, out=4096, bias=True, act="gelu", residual=True,
             pre=True, out_dtype="bf16", dtype="bf16"),
        # its gradient through the activation, and the bias's
        dict(name="act-grad", kind="act_grad", rows=8191, out=4096, act="gelu", dtype="bf16"),
        # gradients of a second product's rows, through the first one's activation, and of its weights
        dict(name="linear-grad", kind="linear_grad", rows=8191, hidden=4096, out=4096, act="silu", residual=False,
             dtype="bf16"),
    ]


# ------------------------------------------------------------------ drawn cases

def _log(rng, lo, hi):
    return int(min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "dropout", "dropout", "linear", "linear", "linear",
                       "act_grad", "linear_grad", "linear_grad"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    case = dict(kind=kind, dtype=dtype)
    if kind in ("norm", "norm_grad", "dropout"):
        case["dtype"] = rng.choice(["bf16", "bf16", "f16", "f32"])
        case["hidden"] = 8 * _log(rng, 8, 1024) if rng.random() < 0.7 else _log(rng, 1, 8192)
        case["tokens"] = min(_log(rng, 1, 16384), max(1, (1 << 26) // case["hidden"]))
        if kind == "dropout":
            case.update(p=round(rng.uniform(0.0, 0.6), 3), residual=rng.random() < 0.5)
        else:
            case.update(center=rng.random() < 0.6, affine=rng.choice(["wb", "wb", "w", "none"]),
                        params=rng.choice(["f32", case["dtype"]]))
            if kind == "norm_grad":
                case["residual"] = rng.random() < 0.5
        return case
    if kind == "act_grad":
        case.update(out=8 * _log(rng, 8, 1024), act=rng.choice(ACTS[1:]))
        case["rows"] = min(_log(rng, 1, 16384), max(1, (1 << 26) // case["out"]))
        return case
    # products: widths in steps of eight values, rows of any number
    case.update(hidden=8 * _log(rng, 8, 896), out=8 * _log(rng, 4, 512), act=rng.choice(ACTS), residual=rng.random() < 0.4)
    most = (1 << 37 if kind == "linear" else 1 << 36) // (case["hidden"] * case["out"])
    case["rows"] = min(_log(rng, 1, 16384), max(1, most))
    if kind == "linear":
        case.update(bias=rng.random() < 0.6, pre=rng.random() < 0.3, out_dtype=rng.choice([dtype, dtype, "f32"]))
    return case


# ------------------------------------------------------------------ inputs

def _normal(shape, gen, dtype, std=1.0):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    return out.normal_(0.0, std, generator=gen)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    s = types.SimpleNamespace(case=case, kind=kind)
    if kind in ("norm", "norm_grad"):
        t, h, param = case["tokens"], case["hidden"], DTYPES[case["params"]]
        # a residual stream: tokens of unequal size, some columns far off the others
        column = 1.0 + 4.0 * (torch.rand(h, generator=gen, device="cuda") < 0.02)
        size = torch.exp(0.5 * torch.randn(t, 1, generator=gen, device="cuda"))
        s.x = ((torch.randn(t, h, generator=gen, device="cuda") + 0.3) * column * size).to(dtype)
        s.weight = (1 + _normal((h,), gen, torch.float32, 0.2)).to(param) if "w" in case["affine"] else None
        s.bias = _normal((h,), gen, param, 0.1) if "b" in case["affine"] else None
        s.eps = 1e-5
        if kind == "norm":
            s.out = torch.zeros_like(s.x)
            s.stats = torch.zeros((t, 2), dtype=torch.float32, device="cuda")
            return s
        # the statistics as the forward pass left them
        x = s.x.double()
        mean = x.mean(1) if case["center"] else torch.zeros(t, dtype=torch.float64, device="cuda")
        s.stats = torch.stack([mean, ((x - mean[:, None]).square().mean(1) + s.eps).rsqrt()], 1).float()
        s.d_out = _normal((t, h), gen, dtype)
        s.residual = _normal((t, h), gen, dtype) if case["residual"] else None
        s.d_x = torch.zeros_like(s.x)
        s.d_weight, s.d_bias = (torch.zeros(h, dtype=torch.float32, device="cuda") for _ in range(2))
        return s
    if kind == "dropout":
        t, h = case["tokens"], case["hidden"]
        s.x = _normal((t, h), gen, dtype)
        s.residual = _normal((t, h), gen, dtype) if case["residual"] else None
        s.seed = seed * 0x2545F4914F6CDD1D % (1 << 64)
        s.step = torch.randint(0, 1 << 40, (1,), generator=gen, device="cuda")
        s.out = torch.zeros_like(s.x)
        return s
    if kind == "act_grad":
        r, n = case["rows"], case["out"]
        s.dy, s.pre = _normal((r, n), gen, dtype), _normal((r, n), gen, dtype, 1.5)
        s.out = torch.zeros_like(s.dy)
        s.d_bias = torch.zeros(n, dtype=torch.float32, device="cuda")
        return s
    r, k, n = case["rows"], case["hidden"], case["out"]
    s.x = _normal((r, k), gen, dtype)
    s.w = _normal((n, k), gen, dtype, k ** -0.5)
    if kind == "linear":
        wide = DTYPES[case["out_dtype"]]
        s.bias = _normal((n,), gen, torch.float32, 0.5) if case["bias"] else None
        s.residual = _normal((r, n), gen, wide) if case["residual"] else None
        s.out = torch.zeros((r, n), dtype=wide, device="cuda")
        s.pre = torch.zeros((r, n), dtype=dtype, device="cuda") if case["pre"] else None
        return s
    s.dy = _normal((r, n), gen, dtype)
    s.pre = _normal((r, k), gen, dtype, 1.5) if case["act"] != "none" else None
    s.residual = _normal((r, k), gen, dtype) if case["residual"] else None
    s.d_x = torch.zeros_like(s.x)
    s.d_w = torch.zeros((n, k), dtype=torch.float32, device="cuda")
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2609_34340_amd as vp
    kind, case = s.kind, s.case
    if kind == "norm":
        vp.layer_norm(s.x, s.weight, s.bias, eps=s.eps, center=case["center"], out=s.out, stats=s.stats)
        return dict(out=s.out, stats=s.stats)
    if kind == "norm_grad":
        vp.layer_norm_grad(s.d_out, s.x, s.stats, s.weight, center=case["center"], residual=s.residual, d_x=s.d_x,
                           d_weight=s.d_weight, d_bias=s.d_bias)
        return dict(d_x=s.d_x, d_weight=s.d_weight, d_bias=s.d_bias)
    if kind == "dropout":
        return vp.dropout(s.x, case["p"], s.seed, step=s.step, residual=s.residual, out=s.out)
    if kind == "act_grad":
        vp.linear_act_grad(s.dy, s.pre, act=case["act"], out=s.out, d_bias=s.d_bias)
        return dict(d_pre=s.out, d_bias=s.d_bias)
    if kind == "linear":
        vp.linear(s.x, s.w, s.bias, act=case["act"], residual=s.residual, out=s.out, pre=s.pre)
        return dict(out=s.out) if s.pre is None else dict(out=s.out, pre=s.pre)
    vp.linear_grad_x(s.dy, s.w, act=case["act"], pre=s.pre, residual=s.residual, out=s.d_x)
    vp.linear_grad_w(s.dy, s.x, out=s.d_w)
    return dict(d_x=s.d_x, d_w=s.d_w)


def _run_plain(s):
    kind, case = s.kind, s.case
    if kind == "norm":
        x = s.x.float()
        mean = x.mean(1, keepdim=True) if case["center"] else torch.zeros((x.shape[0], 1), device=x.device)
        d = x - mean
        rstd = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + s.eps)
        y = d * rstd
        y = y if s.weight is None else y * s.weight.float()
        y = y if s.bias is None else y + s.bias.float()
        return dict(out=y.to(s.x.dtype), stats=torch.cat([mean, rstd], 1))
    if kind == "norm_grad":
        mean, rstd = s.stats[:, :1], s.stats[:, 1:]
        unit = (s.x.float() - mean) * rstd
        dy = s.d_out.float()
        g = dy if s.weight is None else dy * s.weight.float()
        dx = g - unit * (g * unit).mean(1, keepdim=True)
        if case["center"]:
            dx = dx - g.mean(1, keepdim=True)
        dx = dx * rstd
        if s.residual is not None:
            dx = dx + s.residual.float()
        return dict(d_x=dx.to(s.x.dtype), d_weight=(dy * unit).sum(0), d_bias=dy.sum(0))
    if kind == "dropout":
        kept, scale = _kept(s)
        y = torch.where(kept, s.x.float() * scale, 0.0)
        if s.residual is not None:
            y = y + s.residual.float()
        return y.to(s.x.dtype)
    if kind == "act_grad":
        d = s.dy.float() * _slope(s.pre.float(), case["act"])
        return dict(d_pre=d.to(s.dy.dtype), d_bias=d.sum(0))
    if kind == "linear":
        z = s.x.float() @ s.w.float().t()
        if s.bias is not None:
            z = z + s.bias
        y = _act(z, case["act"])
        if s.residual is not None:
            y = y + s.residual.float()
        y = y.to(s.out.dtype)
        return dict(out=y) if s.pre is None else dict(out=y, pre=z.to(s.x.dtype))
    dy = s.dy.float()
    dx = dy @ s.w.float()
    if s.pre is not None:
        dx = dx * _slope(s.pre.float(), case["act"])
    if s.residual is not None:
        dx = dx + s.residual.float()
    return dict(d_x=dx.to(s.x.dtype), d_w=dy.t() @ s.x.float())


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z * z * z)))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "silu":
        q = 1 / (1 + torch.exp(-z))
        return q * (1 + z * (1 - q))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    if act == "gelu_tanh":
        c = (2 / math.pi) ** 0.5
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _signed(v):
    v %= 1 << 64
    return v - (1 << 64) if v >> 63 else v


def _mix(z):
    """SplitMix64's output function on int64 tensors, whose products wrap."""
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * _signed(MIX1)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * _signed(MIX2)
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _kept(s):
    """Which values stay, and their factor: four neighbouring values of a row share a 64-bit word of a SplitMix64 stream
    whose state follows from seed and step, 16 bits each, and stay where these reach p 2^16."""
    (t, h), p = s.x.shape, s.case["p"]
    first = _mix(torch.full((1,), _signed(s.seed + GAMMA), device="cuda", dtype=torch.int64))
    key = _mix((first ^ s.step) + _signed(GAMMA))
    words = (h + 3) // 4
    n = torch.arange(1, t * words + 1, device="cuda").view(t, words, 1)
    field = _mix(key + n * _signed(GAMMA)) >> torch.arange(0, 64, 16, device="cuda") & 0xffff
    least = math.floor(p * 65536 + 0.5)
    return field.view(t, words * 4)[:, :h] >= least, 65536 / (65536 - least) if least < 65536 else 0.0


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    kind = s.kind
    wide = lambda v: None if v is None else v.double()  # noqa: E731
    if kind in ("norm", "norm_grad"):
        # statistics by torch's reductions; the gradients of weight and bias by differentiation
        x, h = s.x.double(), case["hidden"]
        w = (torch.ones(h, dtype=torch.float64, device="cuda") if s.weight is None else s.weight.double()).requires_grad_()
        b = (torch.zeros(h, dtype=torch.float64, device="cuda") if s.bias is None else s.bias.double()).requires_grad_()
        with torch.enable_grad():
            if kind == "norm_grad":   # the operator takes the statistics that it is given, rounded, as the row's
                mean, rstd = s.stats.double().unbind(1)
                y, back = (x - mean[:, None]) * rstd[:, None], s.d_out.double()
                g = back * w.detach()
                moved = g - y * torch.einsum("th,th->t", g, y)[:, None] / h
                if case["center"]:
                    moved = moved - (g.sum(1) / h)[:, None]
                dx = moved * rstd[:, None]
                if s.residual is not None:
                    dx = dx + s.residual.double()
                d_w, d_b = torch.autograd.grad(y * w + b, (w, b), back)
                return dict(d_x=dx, d_weight=d_w, d_bias=d_b)
            if case["center"]:
                var, mean = torch.var_mean(x, 1, correction=0)
            else:
                mean = torch.zeros(case["tokens"], dtype=torch.float64, device="cuda")
                var = torch.linalg.vector_norm(x, dim=1) ** 2 / h
            rstd = (var + s.eps) ** -0.5
            out = torch.addcmul(b.detach(), (x - mean[:, None]) * rstd[:, None], w.detach())
            return dict(out=out, stats=torch.stack([mean, rstd], 1))
    if kind == "dropout":
        kept, scale = _kept_exact(s)
        y = s.x.double() * scale * kept
        return y if s.residual is None else y + s.residual.double()
    if kind == "act_grad":
        leaf = s.pre.double().requires_grad_()
        with torch.enable_grad():
            d, = torch.autograd.grad(_act_exact(leaf, case["act"]), leaf, s.dy.double())
        return dict(d_pre=d, d_bias=torch.mv(d.t(), torch.ones(len(d), dtype=torch.float64, device="cuda")))
    x, w = s.x.double(), s.w.double()
    if kind == "linear":
        z = torch.mm(x, w.t())
        z = z if s.bias is None else z.add_(s.bias.double())
        y = _act_exact(z, case["act"])
        y = y if s.residual is None else y + s.residual.double()
        return dict(out=y) if s.pre is None else dict(out=y, pre=z)
    dy = s.dy.double()
    dx = torch.mm(dy, w)
    if s.pre is not None:
        leaf = s.pre.double().requires_grad_()
        with torch.enable_grad():
            dx, = torch.autograd.grad(_act_exact(leaf, case["act"]), leaf, dx)
    return dict(d_x=dx if s.residual is None else dx + wide(s.residual), d_w=torch.mm(dy.t(), x))


def _act_exact(z, act):
    """By torch's own functions in 64 bits; the gradients follow from them by differentiation."""
    f = torch.nn.functional
    return {"none": lambda: z * 1.0, "relu": lambda: f.relu(z), "silu": lambda: f.silu(z), "gelu": lambda: f.gelu(z),
            "gelu_tanh": lambda: f.gelu(z, approximate="tanh")}[act]()


def _kept_exact(s):
    """The mask by numpy's unsigned 64-bit integers on the host."""
    import numpy as np

    def mixed(z):
        z = (z ^ (z >> np.uint64(30))) * np.uint64(MIX1)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(MIX2)
        return z ^ (z >> np.uint64(31))

    t, h = s.x.shape
    with np.errstate(over="ignore"):
        gamma = np.uint64(GAMMA)
        key = mixed(np.array([s.seed], dtype=np.uint64) + gamma) ^ s.step.cpu().numpy().astype(np.uint64)
        key = mixed(key + gamma)
        words = (h + 3) // 4
        n = np.arange(t * words, dtype=np.uint64) + np.uint64(1)
        raw = mixed(key + n * gamma)
    field = raw.astype("<u8").view("<u2").reshape(t, words * 4)[:, :h]   # lowest 16 bits first
    least = int(np.floor(s.case["p"] * 65536 + 0.5))
    kept = torch.from_numpy(np.ascontiguousarray(field >= least)).cuda()
    return kept, (1 / (1 - least / 65536) if least < 65536 else 0.0)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    """Inputs read once and outputs written once; two operations for each product's multiply and add, one for each
    value's step of a norm, a mask or an activation."""
    kind, size = case["kind"], DTYPES[case["dtype"]].itemsize
    if kind in ("norm", "norm_grad"):
        t, h = case["tokens"], case["hidden"]
        params = len(case["affine"].replace("none", "")) * h * DTYPES[case["params"]].itemsize
        if kind == "norm":
            return dict(bytes=2 * t * h * size + 8 * t + params, flops=6 * t * h)
        return dict(bytes=(3 + bool(case["residual"])) * t * h * size + 8 * t + params + 8 * h, flops=12 * t * h)
    if kind == "dropout":
        n = case["tokens"] * case["hidden"]
        return dict(bytes=(2 + bool(case["residual"])) * n * size, flops=5 * n)
    if kind == "act_grad":
        n = case["rows"] * case["out"]
        return dict(bytes=3 * n * size + 4 * case["out"], flops=10 * n)
    r, k, n = case["rows"], case["hidden"], case["out"]
    if kind == "linear":
        out = DTYPES[case["out_dtype"]].itemsize
        b = (r * k + n * k + bool(case["pre"]) * r * n) * size + (1 + bool(case["residual"])) * r * n * out
        return dict(bytes=b + 4 * n * bool(case["bias"]), flops=2 * r * k * n)
    extra = (case["act"] != "none") + bool(case["residual"])
    return dict(bytes=(r * n + n * k + (2 + extra) * r * k) * size + 4 * n * k, flops=4 * r * k * n)
