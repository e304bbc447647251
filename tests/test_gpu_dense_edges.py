"""Norm, dropout and dense products where values leave the usual range."""
import math

import pytest
import torch

from test_gpu_dense import normal, vp  # noqa: F401

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
