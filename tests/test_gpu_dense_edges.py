"""Norm and dense products where values leave the usual range, few rows by wide outputs, and results over their
residual."""
import math

import pytest
import torch

import dense_reference as ref
from test_gpu_dense import near, near_rounded, normal, vp  # noqa: F401
from test_gpu_dense_kernels import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=str)
def test_slopes_of_the_largest_values(vp, act, dtype):  # noqa: F811
    """1 and 0 exactly at values whose cube or square passes 32 bits, and at infinities, which a kept value of 16 bits
    rounds to; a NaN stays one."""
    far = torch.tensor([2.0 ** e for e in (7, 15, 30, 43, 63, 64, 66, 100, 127)] + [math.inf]).to(dtype)
    N = 2 * len(far) + 2
    pre = torch.cat([far, -far, torch.full((2,), math.nan, dtype=dtype)]).repeat(3, 1).cuda()
    d = normal((3, N), 1, dtype).cuda()
    got, sums = vp.linear_act_grad(d, pre, act=act)
    n = len(far)
    assert torch.equal(got[:, :n], d[:, :n]) and (got[:, n:2 * n].abs() <= 1e-28).all() and got[:, -2:].isnan().all()
    assert sums[:2 * n].isfinite().all() and sums[-2:].isnan().all()
    if dtype == torch.float32:
        return
    # the same through a product's epilogue, of a tile's and of parts' sums
    for R, K in ((3, 64), (3, 4096)):
        pre = torch.cat([far, -far]).repeat(R, 1).cuda()
        pre = torch.cat([pre, torch.zeros(R, 24 - 2 * n, dtype=dtype, device="cuda")], 1)
        d, w = normal((R, K), 2, dtype).cuda(), normal((K, 24), 3, dtype, 0.1).cuda()
        got, plain = vp.linear_grad_x(d, w, act=act, pre=pre), vp.linear_grad_x(d, w)
        assert torch.equal(got[:, :n], plain[:, :n]) and (got[:, n:2 * n].abs() <= 1e-28).all()


@pytest.mark.parametrize("H", [61, 64, 250, 256, 1277, 1280, 32768])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
def test_gradient_of_equal_values_far_from_zero(vp, H, dtype):  # noqa: F811
    """Rows of one value 2^80 and a tiny eps: m r passes 32 bits, where a row's lanes hold nothing as well, but u is 0 and
    the gradient r (g - mean(g))."""
    x = torch.full((3, H), 2.0 ** 80, dtype=dtype)
    x[1] = 1.0
    want = torch.tensor([[2.0 ** 80, 1e15], [1.0, 1e15], [2.0 ** 80, 1e15]], dtype=torch.float64)
    stats = want.float().cuda()
    # the mean is exact where every wavefront holds a power of two values (of 1280 in 16 bits one holds 768, and 1 / 768 rounds)
    if H in (64, 256, 32768) or (H == 1280 and dtype == torch.float32):
        assert (vp.layer_norm(x.cuda(), eps=1e-30, stats=stats.fill_(math.nan)) == 0).all()
        near(stats, want, 8 * ref.U * want)
    d = normal((3, H), 1, dtype)
    dx, e, dw, e_w, db, e_b = ref.norm_grad(d, x, stats.cpu(), None, True)
    got = vp.layer_norm_grad(d.cuda(), x.cuda(), stats)
    near_rounded(got[0], dx, e)
    near(got[1], dw, e_w + 1e-30)
    near(got[2], db, e_b + 1e-30)


# R, N, K, kernel, parts: None where any number above one does
WIDE = [(33, 57344, 1024, "tiles_128", 1), (64, 28680, 1032, "tiles_alone", 1), (65, 16384, 1024, "tiles_alone", 1), (127, 65544, 1024, "tiles_128", 1),
        (100, 8192, 4104, "tiles_alone", None), (97, 4096, 8192, "tiles_alone", None), (32, 57344, 1024, "few_rows", 1)]


@pytest.mark.parametrize("case", WIDE, ids=lambda c: "-".join(map(str, c)))
def test_few_rows_by_wide_outputs(vp, case):  # noqa: F811
    R, N, K, kernel, parts = case
    kind, n = vp.linear_kernel(R, N, K)
    assert kind == kernel and (n == parts if parts else n > 1)
    check(vp, "forward", R, N, K, torch.bfloat16)


@pytest.mark.parametrize("H", [100, 4096, 20000])
def test_gradient_of_rows_far_from_zero(vp, H):  # noqa: F811
    """Forward statistics into the gradient, against the statistics of 64 bits.  The mean in 32 bits is off by up to half
    a unit of its last place and by the forward's own bound: every u of the row moves by that times r, which the result
    takes once through u and once through mean(g u); r's bound counts three times."""
    x = normal((4, H), 1)
    x[0] += 5000.0
    x[2] -= 3e4
    d = normal((4, H), 2)
    _, _, stats, stats_err = ref.norm(x, None, None, 1e-5, True)
    st = torch.empty(4, 2, device="cuda")
    vp.layer_norm(x.cuda(), stats=st)
    dx, e, dw, e_w, db, e_b = ref.norm_grad(d, x, stats, None, True)
    m, r = stats[:, :1], stats[:, 1:]
    e_r, off = stats_err[:, 1:], stats_err[:, :1] * r   # of r, and of u
    u, g = (x.double() - m) * r, d.double()
    e_u = (off + u.abs() * e_r / r) * 1.01
    mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731
    moved = r * (e_u * mean(g * u).abs() + (u.abs() + e_u) * mean(g.abs() * e_u))
    got = vp.layer_norm_grad(d.cuda(), x.cuda(), st)
    near_rounded(got[0], dx, 1.01 * (e + dx.abs() * e_r / r + moved))
    near(got[1], dw, 1.01 * e_w + (g.abs() * e_u).sum(0))
    near(got[2], db, e_b)


# direction, R, N, K, kernel, parts: None where any number above one does
OVER = [("forward", 3, 136, 72, "few_rows", 1), ("forward", 40, 520, 4096, "few_rows", None), ("forward", 200, 136, 72, "tiles_alone", 1),
        ("forward", 140, 264, 4104, "tiles_alone", None), ("forward", 3000, 2056, 72, "tiles_128", 1), ("forward", 4090, 4088, 392, "tiles_256", 1),
        ("grad_x", 130, 72, 136, "tiles_alone", 1), ("grad_x", 96, 2056, 520, "tiles_alone", None), ("grad_x", 3000, 72, 2056, "tiles_128", 1),
        ("grad_x", 4090, 392, 4088, "tiles_256", 1)]


@pytest.mark.parametrize("case", OVER, ids=lambda c: "-".join(map(str, c)))
def test_results_over_their_residual(vp, case):  # noqa: F811
    """Every kernel writes over the residual what it writes beside it (which other tests hold to 64 bits)."""
    direction, R, N, K, kernel, parts = case
    kind, n = vp.linear_kernel(R, N, K, direction)
    assert kind == kernel and (n == parts if parts else n > 1)
    x, w, dy = (normal(s, i, torch.bfloat16, std).cuda() for i, (s, std) in enumerate((((R, K), 1.0), ((N, K), 0.1), ((R, N), 1.0))))
    if direction == "forward":
        for dtype in (torch.bfloat16, torch.float32):
            res = normal((R, N), 5, dtype).cuda()
            want = vp.linear(x, w, act="gelu", residual=res, dtype=dtype)
            assert vp.linear(x, w, act="gelu", residual=res, out=res) is res and torch.equal(res, want)
    else:
        res, pre = normal((R, K), 5, torch.bfloat16).cuda(), normal((R, K), 6, torch.bfloat16).cuda()
        want = vp.linear_grad_x(dy, w, act="silu", pre=pre, residual=res)
        assert vp.linear_grad_x(dy, w, act="silu", pre=pre, residual=res, out=res) is res and torch.equal(res, want)


def test_infinite_sums_through_activations(vp):  # noqa: F811
    """Plus infinity stays, minus infinity is relu's 0 and NaN where it meets a factor of 0, and columns keep to themselves."""
    for R, N in ((3, 64), (200, 136)):
        x, w, b = torch.zeros(R, 72, dtype=torch.bfloat16), normal((N, 72), 1, torch.bfloat16), normal((N,), 2)
        b[3], b[N - 1] = math.inf, -math.inf
        for act in ref.ACTS:
            for dtype in (torch.bfloat16, torch.float32):
                got = vp.linear(x.cuda(), w.cuda(), b.cuda(), act=act, dtype=dtype).cpu()
                assert (got[:, 3] == math.inf).all()
                last = got[:, N - 1]
                assert (last == -math.inf).all() if act == "none" else (last == 0).all() if act == "relu" else last.isnan().all()
                assert got[:, :3].isfinite().all() and got[:, 4:N - 1].isfinite().all()


@pytest.mark.parametrize("H", [40, 200, 3000, 40000])
def test_rows_past_the_range_keep_to_themselves(vp, H):  # noqa: F811
    """Finite rows whose squares, or whose sum, pass 2^128: r is 0 or NaN, and the rows beside them are what they were."""
    x = normal((5, H), 1)
    x[1] *= 1e25
    x[3] = 3e38
    for center in (True, False):
        y, err, stats, stats_err = ref.norm(x[::2], None, None, 1e-5, center)
        st = torch.empty(5, 2, device="cuda")
        got = vp.layer_norm(x.cuda(), center=center, stats=st)
        near_rounded(got[::2], y, err)
        near(st[::2], stats, stats_err + 1e-30)
        r = st[1::2, 1]
        assert (r.isnan() | (r == 0)).all()
