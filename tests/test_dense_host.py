"""Refusals of the dense operators before anything is enqueued, and the generator of the mask (no GPU)."""
import math

import numpy as np
import pytest
import torch

import dense_reference as ref

P = 4096   # an aligned address that no refused call touches


@pytest.fixture(scope="module")
def vp():
    import os
    import paper_2609_34340_amd as vp
    if not os.path.exists(vp.LIB_PATH):
        from paper_2609_34340_amd import build
        build.build()
    return vp


def norm(vp, x=P, dtype=1, T=4, H=64, xs=128, w=P, b=P, pd=0, eps=1e-5, center=1, y=P, ys=128, stats=P):
    return vp.lib().vp_layer_norm(x, dtype, T, H, xs, w, b, pd, eps, center, y, ys, stats, None)


def test_layer_norm_refuses(vp):
    bad, far = vp.INVALID_ARGUMENT, vp.UNSUPPORTED
    for kw, status in ((dict(dtype=3), bad), (dict(dtype=-1), bad), (dict(T=-1), bad), (dict(H=0), bad), (dict(H=-8), bad),
                       (dict(xs=126), bad), (dict(xs=129), bad), (dict(ys=120), bad), (dict(x=P + 1), bad), (dict(y=P + 1), bad),
                       (dict(x=None), bad), (dict(y=None), bad), (dict(pd=2), bad), (dict(pd=5), bad), (dict(w=P + 2), bad),
                       (dict(b=P + 1, pd=1), bad), (dict(stats=P + 2), bad), (dict(eps=-1e-9), bad), (dict(eps=math.nan), bad),
                       (dict(eps=math.inf), bad), (dict(center=2), bad), (dict(T=1 << 31), far),
                       (dict(H=(1 << 20) + 1, xs=1 << 22, ys=1 << 22), far)):
        assert norm(vp, **kw) == status, kw
    assert norm(vp, T=0) == vp.OK and norm(vp, T=0, x=None, y=None, stats=None, w=None, b=None) == vp.OK


def norm_grad(vp, d=P, ds=128, x=P, xs=128, dtype=1, T=4, H=64, stats=P, w=P, pd=0, center=1, r=None, rs=0, o=P, os=128,
              dw=P, db=P, ws=P, wb=1 << 20):
    return vp.lib().vp_layer_norm_grad(d, ds, x, xs, dtype, T, H, stats, w, pd, center, r, rs, o, os, dw, db, ws, wb, None)


def test_layer_norm_grad_refuses(vp):
    bad, far = vp.INVALID_ARGUMENT, vp.UNSUPPORTED
    need = vp.layer_norm_grad_workspace_bytes(4, 64)
    assert need > 0 and vp.layer_norm_grad_workspace_bytes(-1, 64) == 0 and vp.layer_norm_grad_workspace_bytes(4, 0) == 0
    for kw, status in ((dict(dtype=4), bad), (dict(T=-1), bad), (dict(H=0), bad), (dict(d=None), bad), (dict(x=None), bad),
                       (dict(o=None), bad), (dict(stats=None), bad), (dict(stats=P + 1), bad), (dict(ds=64), bad), (dict(xs=127), bad),
                       (dict(os=2), bad), (dict(r=P, rs=64), bad), (dict(r=P + 1, rs=128), bad), (dict(pd=2), bad), (dict(w=P + 2), bad),
                       (dict(dw=P + 2), bad), (dict(db=P + 1), bad), (dict(ws=None), bad), (dict(ws=P + 8), bad), (dict(wb=need - 1), bad),
                       (dict(center=-1), bad), (dict(T=1 << 31), far), (dict(H=1 << 21, xs=1 << 22, ds=1 << 22, os=1 << 22), far)):
        assert norm_grad(vp, **kw) == status, kw


def test_dropout_refuses(vp):
    bad, far = vp.INVALID_ARGUMENT, vp.UNSUPPORTED

    def drop(x=P, dtype=2, T=4, H=64, xs=128, p=0.5, step=None, r=None, rs=0, o=P, os=128):
        return vp.lib().vp_dropout(x, dtype, T, H, xs, p, 1, step, r, rs, o, os, None)
    for kw, status in ((dict(dtype=7), bad), (dict(T=-1), bad), (dict(H=0), bad), (dict(p=-1e-9), bad), (dict(p=1.0000001), bad),
                       (dict(p=math.nan), bad), (dict(x=None), bad), (dict(o=None), bad), (dict(step=P + 4), bad), (dict(xs=127), bad),
                       (dict(os=126), bad), (dict(r=P, rs=2), bad), (dict(o=P + 1), bad), (dict(T=1 << 31), far),
                       (dict(H=1 << 21, xs=1 << 22, os=1 << 22), far)):
        assert drop(**kw) == status, kw
    assert drop(T=0, x=None, o=None) == vp.OK


def linear(vp, x=P, xs=128, dtype=1, w=P, wst=128, R=4, N=32, K=64, b=P, bd=0, act=0, r=None, rs=0, y=P, od=1, ys=64, pre=None,
           ps=0, ws=P, wb=1 << 30):
    return vp.lib().vp_linear(x, xs, dtype, w, wst, R, N, K, b, bd, act, r, rs, y, od, ys, pre, ps, ws, wb, None)


def grad_x(vp, d=P, ds=64, dtype=1, w=P, wst=128, R=4, N=32, K=64, act=0, pre=None, ps=0, r=None, rs=0, o=P, os=128, ws=P, wb=1 << 30):
    return vp.lib().vp_linear_grad_x(d, ds, dtype, w, wst, R, N, K, act, pre, ps, r, rs, o, os, ws, wb, None)


def grad_w(vp, d=P, ds=64, x=P, xs=128, dtype=1, R=4, N=32, K=64, o=P, ws=P, wb=1 << 30):
    return vp.lib().vp_linear_grad_w(d, ds, x, xs, dtype, R, N, K, o, ws, wb, None)


SIZES = [(dict(R=-1), 1), (dict(N=0), 1), (dict(K=0), 1), (dict(N=12), 5), (dict(K=60), 5), (dict(dtype=0), 1), (dict(dtype=3), 1),
         (dict(R=1 << 31), 5), (dict(N=(1 << 20) + 8), 5), (dict(K=(1 << 20) + 8), 5)]


def test_linear_refuses(vp):
    bad, far = vp.INVALID_ARGUMENT, vp.UNSUPPORTED
    assert (bad, far) == (1, 5)
    for kw, status in SIZES + [
            (dict(x=None), bad), (dict(w=None), bad), (dict(y=None), bad), (dict(x=P + 8), bad), (dict(w=P + 2), bad), (dict(y=P + 4), bad),
            (dict(xs=120), bad), (dict(xs=136), bad), (dict(wst=64), bad), (dict(ys=72), bad), (dict(ys=48), bad), (dict(act=5), bad),
            (dict(act=-1), bad), (dict(od=2), bad), (dict(od=0, ys=64), bad), (dict(bd=2), bad), (dict(b=P + 4), bad), (dict(r=P, rs=32), bad),
            (dict(pre=P, ps=32), bad), (dict(pre=P + 8, ps=64), bad), (dict(xs=(1 << 22) + 16), far), (dict(wst=(1 << 22) + 16), far),
            (dict(ys=(1 << 22) + 16), far)]:
        assert linear(vp, **kw) == status, kw
    assert linear(vp, R=0, x=None, y=None) == vp.OK


def test_linear_gradients_refuse(vp):
    bad, far = vp.INVALID_ARGUMENT, vp.UNSUPPORTED
    for kw, status in SIZES + [
            (dict(d=None), bad), (dict(w=None), bad), (dict(o=None), bad), (dict(ds=48), bad), (dict(wst=120), bad), (dict(os=100), bad),
            (dict(act=3), bad), (dict(pre=P, ps=128), bad), (dict(act=3, pre=P, ps=64), bad), (dict(act=9, pre=P, ps=128), bad),
            (dict(r=P, rs=64), bad), (dict(ds=(1 << 22) + 16), far)]:
        assert grad_x(vp, **kw) == status, kw
    assert grad_x(vp, R=0, d=None, o=None) == vp.OK
    for kw, status in SIZES + [(dict(d=None), bad), (dict(x=None), bad), (dict(o=None), bad), (dict(o=P + 4), bad), (dict(ds=32), bad),
                               (dict(xs=(1 << 22) + 16), far)]:
        assert grad_w(vp, **kw) == status, kw


def test_linear_workspaces(vp):
    for direction, call in (("forward", linear), ("grad_x", grad_x), ("grad_w", grad_w)):
        for R, N, K in ((96, 256, 7168), (4, 32, 64), (16384, 256, 4096), (64, 4096, 4096)):
            need = vp.linear_workspace_bytes(R, N, K, direction)
            assert need % 16 == 0
            sizes = dict(R=R, N=N, K=K)
            if direction == "forward":
                sizes.update(xs=2 * K, wst=2 * K, ys=2 * N)
            elif direction == "grad_x":
                sizes.update(ds=2 * N, wst=2 * K, os=2 * K)
            else:
                sizes.update(ds=2 * N, xs=2 * K)
            if need:
                assert call(vp, wb=need - 1, **sizes) == vp.INVALID_ARGUMENT
                assert call(vp, ws=None, wb=0, **sizes) == vp.INVALID_ARGUMENT
                assert call(vp, ws=P + 8, **sizes) == vp.INVALID_ARGUMENT
    assert vp.lib().vp_linear_workspace(3, 96, 256, 7168) == 0 and vp.lib().vp_linear_workspace(0, 96, 12, 7168) == 0


def test_linear_act_grad_refuses(vp):
    bad, far = vp.INVALID_ARGUMENT, vp.UNSUPPORTED
    need = vp.linear_act_grad_workspace_bytes(4, 64)

    def call(d=P, ds=128, pre=P, ps=128, dtype=1, R=4, N=64, act=2, o=P, os=128, db=P, ws=P, wb=1 << 20):
        return vp.lib().vp_linear_act_grad(d, ds, pre, ps, dtype, R, N, act, o, os, db, ws, wb, None)
    for kw, status in ((dict(dtype=3), bad), (dict(R=-1), bad), (dict(N=0), bad), (dict(act=5), bad), (dict(pre=None), bad), (dict(act=0), bad),
                       (dict(o=None, db=None), bad), (dict(d=None), bad), (dict(ds=64), bad), (dict(ps=64), bad), (dict(os=127), bad),
                       (dict(db=P + 2), bad), (dict(ws=None), bad), (dict(wb=need - 1), bad), (dict(R=1 << 31), far),
                       (dict(N=1 << 21, ds=1 << 22, ps=1 << 22, os=1 << 22), far)):
        assert call(**kw) == status, kw
    assert call(R=0, db=None, d=None, pre=None, o=P) == vp.OK


def test_the_binding_refuses(vp):
    """What the checks of tensors refuse before the library is called (tensors of the CPU are refused first)."""
    x = torch.zeros(2, 16, dtype=torch.bfloat16)
    for f in (lambda: vp.layer_norm(x), lambda: vp.dropout(x, 0.5, 1), lambda: vp.linear(x, x), lambda: vp.linear_act_grad(x),
              lambda: vp.linear_grad_x(x, x), lambda: vp.linear_grad_w(x, x), lambda: vp.layer_norm_grad(x, x, x)):
        with pytest.raises(ValueError):
            f()
    from paper_2609_34340_amd.dense import _act
    with pytest.raises(ValueError):
        _act("tanh")
    assert [_act(a) for a in ref.ACTS] == [0, 1, 2, 3, 4]


def test_the_masks_generator_is_splitmix64():
    """Outputs of state 0 as published with the generator, and the mask's words by its recurrence written with integers."""
    with np.errstate(over="ignore"):
        out = ref.mixed(np.arange(1, 4, dtype=np.uint64) * ref.GAMMA)
    assert [int(v) for v in out] == [0xE220A8397B1DCDAF, 0x6E789E6AA1B965F4, 0x06C45D188009454F]
    M = (1 << 64) - 1

    def mix(z):
        z = (z ^ z >> 30) * 0xBF58476D1CE4E5B9 & M
        z = (z ^ z >> 27) * 0x94D049BB133111EB & M
        return z ^ z >> 31
    g, seed, step, T, H, p = 0x9E3779B97F4A7C15, (1 << 64) - 2, -7, 3, 6, 0.3
    state = mix((mix(seed + g & M) ^ (step & M)) + g & M)
    mask, scale = ref.kept(T, H, p, seed, step)
    least = round(65536 * p)
    for t in range(T):
        for c in range(H):
            word = mix(state + (t * 2 + c // 4 + 1) * g & M)
            assert bool(mask[t, c]) == (word >> 16 * (c % 4) & 0xffff >= least)
    assert scale == 65536 / (65536 - least)


def test_the_references_slopes_against_differences():
    v = torch.linspace(-9, 9, 4001, dtype=torch.float64)[1::2]   # without 0
    h = 1e-5
    for name in ref.ACTS:
        if name == "relu":
            assert torch.equal(ref.slope(v, name), (v > 0).double())
            continue
        d = (ref.act(v + h, name) - ref.act(v - h, name)) / (2 * h)
        assert (d - ref.slope(v, name)).abs().max() < 1e-8   # h^2 / 6 of third derivatives below 3, and 1e-16 |v| / h
        assert (ref.act(v, name) - {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu,
                                    "gelu_tanh": lambda u: torch.nn.functional.gelu(u, approximate="tanh"),
                                    "none": lambda u: u}[name](v)).abs().max() < 1e-14
