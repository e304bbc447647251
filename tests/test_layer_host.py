"""Refusals of the layer operators before anything is enqueued, and the tests' own 64-bit reference (no GPU)."""
import ctypes as C
import math

import pytest
import torch

import layer_reference as ref


@pytest.fixture(scope="module")
def vp():
    import os
    import paper_2609_34340_amd as vp
    if not os.path.exists(vp.LIB_PATH):
        from paper_2609_34340_amd import build
        build.build()
    return vp


P = 4096   # an aligned address that no refused call touches


def params(vp, **kw):
    from paper_2609_34340_amd.layer import RouteParams
    d = dict(score=0, top_k=8, n_groups=1, top_groups=1, group_top=1, renorm=1, scale=1.0)
    d.update(kw)
    return RouteParams(*[d[f] for f, _ in RouteParams._fields_])


@pytest.mark.parametrize("kw,status", [
    (dict(top_k=0), 1), (dict(top_k=65), 5), (dict(top_k=257), 1), (dict(score=2), 1), (dict(n_groups=0), 1),
    (dict(n_groups=3), 1), (dict(n_groups=8, top_groups=9), 1), (dict(n_groups=8, top_groups=0), 1),
    (dict(n_groups=64, top_groups=1), 1), (dict(n_groups=128, top_groups=64), 5), (dict(group_top=3), 1),
    (dict(renorm=2), 1), (dict(scale=0.0), 1), (dict(scale=-1.0), 1), (dict(scale=math.inf), 1), (dict(scale=math.nan), 1)])
def test_route_refuses(vp, kw, status):
    L = vp.lib()
    p = params(vp, **kw)
    assert L.vp_route(P, 0, 4, 256, 256, C.byref(p), None, P, P, None) == status
    assert L.vp_route_grad(P, 0, 4, 256, 256, C.byref(p), P, P, P, P, P, None) == status


def test_route_refuses_sizes_and_pointers(vp):
    L, p = vp.lib(), params(vp)
    bad = vp.INVALID_ARGUMENT
    assert L.vp_route(P, 3, 4, 256, 256, C.byref(p), None, P, P, None) == bad        # element type
    assert L.vp_route(P, 0, -1, 256, 256, C.byref(p), None, P, P, None) == bad
    assert L.vp_route(P, 0, 4, 256, 255, C.byref(p), None, P, P, None) == bad        # rows overlap
    assert L.vp_route(P, 0, 4, 4104, 4104, C.byref(p), None, P, P, None) == vp.UNSUPPORTED
    assert L.vp_route(P, 0, 1 << 28, 256, 256, C.byref(p), None, P, P, None) == vp.UNSUPPORTED
    assert L.vp_route(P, 0, 4, 256, 256, None, None, P, P, None) == bad
    for args in ((None, P, P), (P, None, P), (P, P, None)):
        assert L.vp_route(args[0], 0, 4, 256, 256, C.byref(p), None, args[1], args[2], None) == bad
    assert L.vp_route_grad(P, 0, 4, 256, 256, C.byref(p), P, P, P, None, P, None) == bad
    assert L.vp_route_grad(P, 0, 0, 256, 256, C.byref(p), P, P, P, P, None, None) == vp.OK   # no status, no report
    assert L.vp_expert_offsets(P, 3, 8, 0, P, P, None) == bad
    assert L.vp_expert_offsets(P, 2, 8, 2, P, P, None) == bad
    assert L.vp_expert_offsets(P, 2, 8192, 0, P, P, None) == bad
    assert L.vp_expert_offsets(None, 2, 8, 0, P, P, None) == bad


def matmul(vp, **kw):
    d = dict(x=P, x_stride=128, dtype=1, w=P, off=P, R=4, L=2, N=32, K=64, gated=0, y=P, y_stride=64, pre=None,
             pre_stride=0, st=P, stream=None)
    d.update(kw)
    return vp.lib().vp_expert_matmul(*d.values())


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=0), 1), (dict(dtype=7), 1), (dict(R=-1), 1), (dict(L=0), 1), (dict(L=4097), 5), (dict(N=12), 5),
    (dict(K=60), 5), (dict(N=0), 1), (dict(K=0), 1), (dict(x=None), 1), (dict(w=None), 1), (dict(y=None), 1),
    (dict(off=None), 1), (dict(x=P + 8), 1), (dict(w=P + 2), 1), (dict(y=P + 4), 1),
    (dict(x_stride=120), 1), (dict(x_stride=136), 1), (dict(y_stride=48), 1), (dict(x_stride=(1 << 22) + 16), 5),
    (dict(gated=2), 1), (dict(gated=1, N=24), 5), (dict(pre=P, pre_stride=64), 1), (dict(gated=1, pre=P, pre_stride=32), 1),
    (dict(R=1 << 31), 5), (dict(K=1 << 21, x_stride=1 << 22), 5)])
def test_expert_matmul_refuses(vp, kw, status):
    assert matmul(vp, **kw) == status


def test_no_rows_is_no_error(vp):
    assert matmul(vp, R=0, x=None, y=None) == vp.OK
    assert matmul(vp, R=0, x=None, y=None, st=None) == vp.OK
    assert vp.lib().vp_expert_matmul_grad_x(None, 64, 1, P, P, 0, 2, 32, 64, None, 128, P, None) == vp.OK


def test_other_products_refuse(vp):
    L, bad = vp.lib(), vp.INVALID_ARGUMENT
    assert L.vp_expert_matmul_grad_x(P, 62, 1, P, P, 4, 2, 32, 64, P, 128, P, None) == bad
    assert L.vp_expert_matmul_grad_x(P, 64, 1, P, P, 4, 2, 32, 64, P, 64, P, None) == bad
    assert L.vp_expert_matmul_grad_w(P, 64, P, 128, 1, P, 4, 2, 32, 64, None, P, None) == bad
    assert L.vp_expert_matmul_grad_w(P, 64, P, 128, 0, P, 4, 2, 32, 64, P, P, None) == bad
    assert L.vp_expert_gate_grad(P, 64, P, 64, 1, P, 4, 2, 32, P, 128, P, None) == bad
    assert L.vp_expert_gate_grad(P, 64, P, 128, 1, P, 4, 2, 28, P, 128, P, None) == vp.UNSUPPORTED
    rb = L.vp_mx_row_bytes(64)
    assert L.vp_expert_matmul_mx(P, rb, P, P, 4, 2, 32, 48, 0, P, 1, 64, P, None) == vp.UNSUPPORTED
    assert L.vp_expert_matmul_mx(P, rb - 16, P, P, 4, 2, 32, 64, 0, P, 1, 64, P, None) == bad
    assert L.vp_expert_matmul_mx(P, rb, P, P, 4, 2, 32, 64, 0, P, 0, 64, P, None) == bad


def test_merge_refuses(vp):
    L, bad = vp.lib(), vp.INVALID_ARGUMENT
    ok = dict(rows=P, dtype=1, T=4, k=2, H=64, stride=128, w=P, res=None, res_stride=0, out=P, out_stride=128, stream=None)
    for kw in (dict(dtype=9), dict(T=-1), dict(k=0), dict(k=256), dict(H=0), dict(H=60), dict(stride=112), dict(stride=136),
               dict(rows=None), dict(w=None), dict(out=None), dict(rows=P + 2), dict(out=P + 8), dict(res=P, res_stride=64)):
        assert L.vp_merge(*{**ok, **kw}.values()) == bad, kw
    assert L.vp_merge(*{**ok, "T": 0}.values()) == vp.OK
    assert L.vp_merge(*{**ok, "H": 1 << 21, "stride": 1 << 22, "out_stride": 1 << 22}.values()) == vp.UNSUPPORTED
    assert L.vp_merge_grad(P, 1, 4, 2, 64, 128, P, 128, P, P, 128, None, None) == bad
    assert L.vp_merge_grad(P, 1, 4, 2, 64, 120, P, 128, P, P, 128, P, None) == bad


def test_mx_refuses(vp):
    L, bad = vp.lib(), vp.INVALID_ARGUMENT
    assert [vp.mx_row_bytes(k) for k in (0, -32, 31, 48, 32, 64, 512, 7168)] == [0, 0, 0, 0, 32, 48, 272, 3808]
    assert L.vp_mx_quantize(P, 1, 4, 48, 96, P, 48, None) == vp.UNSUPPORTED
    assert L.vp_mx_quantize(P, 5, 4, 64, 128, P, 48, None) == bad
    assert L.vp_mx_quantize(P, 1, 4, 64, 112, P, 48, None) == bad
    assert L.vp_mx_quantize(P, 1, 4, 64, 128, P, 32, None) == bad
    assert L.vp_mx_quantize(P, 1, 4, 64, 128, None, 48, None) == bad
    assert L.vp_mx_dequantize(P, 4, 64, 48, P + 4, 1, 128, None) == bad
    assert L.vp_mx_dequantize(P, 4, 64, 48, P, 0, 128, None) == bad   # fp32 rows are 256 bytes


def test_python_refuses_what_it_is_given(vp):
    x = torch.zeros(4, 64)
    for call in (lambda: vp.route(x, 2), lambda: vp.expert_matmul(x.bfloat16(), x.view(1, 4, 64).bfloat16(), torch.zeros(2)),
                 lambda: vp.merge(x, torch.zeros(2, 2)), lambda: vp.mx_quantize(x), lambda: vp.expert_offsets(torch.zeros(2, 4), 0),
                 lambda: vp.merge_grad(x, x, torch.zeros(2)), lambda: vp.mx_dequantize(x, 64)):
        with pytest.raises(ValueError):
            call()


def test_reference_levels_by_hand():
    x = torch.zeros(1, 32)
    x[0, :8] = torch.tensor([4.0, 0.25, 0.75, 2.5, 5.0, 7.0, -1.75, 0.2])
    assert ref.mx_values(x)[0, :8].tolist() == [4.0, 0.0, 1.0, 2.0, 4.0, 6.0, -2.0, 0.0]


def test_reference_route_by_hand():
    x = torch.tensor([[1.0, 3.0, 3.0, -math.inf]])
    ids, w, _ = ref.route(x, 3, renorm=True)
    assert ids.tolist() == [[1, 2, 0]]
    e = math.exp(-2.0)
    assert torch.allclose(w, torch.tensor([[1 / (2 + e), 1 / (2 + e), e / (2 + e)]], dtype=torch.float64))
