"""The layer calls where an input is out of the ordinary: values that are no numbers, weights of zero, offsets out of
order, launches of more than 2^32 threads, other streams."""
import math

import pytest
import torch

import layer_reference as ref
from test_gpu_layer import near, normal

pytestmark = pytest.mark.gpu

HALVES = [torch.bfloat16, torch.float16]
FLOATS = HALVES + [torch.float32]


@pytest.fixture(scope="module")
def vp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_34340_amd as vp
    return vp


# ---------------------------------------------------------------- routing

def test_a_scale_that_changed_in_place(vp):
    x, scale = normal((4, 16), 200).cuda(), torch.tensor(1.0)
    one = vp.route(x, 4, scale=scale)
    scale.fill_(2.5)
    got = vp.route(x, 4, scale=scale)
    assert torch.equal(got["ids"], one["ids"])
    near(got["weights"], 2.5 * one["weights"].double().cpu(), 1e-6 * torch.ones(4, 4))
    near(vp.route_grad(x, one["ids"], got["weights"], torch.ones(4, 4).cuda(), renorm=False, scale=scale),
         vp.route_grad(x, one["ids"], got["weights"], torch.ones(4, 4).cuda(), renorm=False, scale=2.5).double().cpu(),
         torch.zeros(4, 16))


@pytest.mark.parametrize("T,E", [(3, 40), (4099, 40), (3, 256), (4099, 256), (3, 1024), (2, 1280)])
@pytest.mark.parametrize("groups", [1, 8])
@pytest.mark.parametrize("dtype", FLOATS, ids=str)
def test_logits_that_are_no_numbers_do_not_decide(vp, T, E, groups, dtype):
    """A softmax's NaN is in every score of its row; the choice is that of the row's numbers all the same."""
    k = 6
    x = normal((T, E), 201, std=2.0).to(dtype)
    x[:, 0], x[:, 1], x[:, 3] = math.nan, -math.inf, math.nan
    x[0, 5] = math.inf
    x[1] = math.nan
    x[1, 7] = 0.5
    bias = 0.01 * normal((E,), 202)
    for b in (bias, None):
        if b is None and groups == 1:
            continue   # the logits decide themselves
        how = dict(bias=None if b is None else b.cuda(), n_groups=groups, top_groups=max(groups // 2, 1), group_top=2)
        got = vp.route(x.cuda(), k, **how)
        ids = got["ids"].cpu().long()
        assert torch.isnan(got["weights"][:, 0]).all()
        clean = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
        if T > 2:   # a row of numbers, masked and not: the same choice as with the others masked
            assert torch.equal(ids[2:], vp.route(clean.cuda(), k, **how)["ids"].cpu().long()[2:])
        assert ids[0, 0] == 5 and not (set(ids[0, 1:].tolist()) & {0, 1, 3})   # infinity is the largest
        assert ids[1, 0] == 7 and ids[1, 1:].tolist() == [0, 1, 2, 3, 4]      # then nothing is left
        assert all(len(set(r.tolist())) == k for r in ids)


@pytest.mark.parametrize("T,E", [(33, 40), (4101, 40), (4101, 256), (9, 1280)])
def test_a_row_with_a_nan_beside_rows_of_numbers(vp, T, E):
    """Tokens that share a wavefront: each is routed as if it were alone."""
    x = normal((T, E), 205, std=2.0)
    odd = torch.arange(T) % 3 == 1
    x[odd, 2], x[odd, 9] = math.nan, math.inf
    x[::7, 4] = -math.inf
    how = dict(bias=0.01 * normal((E,), 206).cuda(), n_groups=8, top_groups=5, group_top=2)
    got = vp.route(x.cuda(), 5, **how)
    for rows in (odd, ~odd):
        alone = vp.route(x[rows].cuda(), 5, **how)
        assert torch.equal(got["ids"][rows.cuda()], alone["ids"])
        assert torch.equal(got["weights"][rows.cuda()].isnan(), alone["weights"].isnan())
    assert torch.isfinite(got["weights"][(~odd).cuda()]).all() and (got["ids"].cpu()[odd][:, 0] == 9).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_a_weight_of_zero_passes_no_gradient_on(vp, score, renorm):
    """Whatever the gradient at a slot of weight 0 is, it does not reach the other slots'."""
    x = normal((2, 12), 203)
    x[:, 3:] = -math.inf   # three experts are left for five slots
    out = vp.route(x.cuda(), 5, score=score, renorm=renorm)
    assert (out["weights"][:, 3:] == 0).all()
    d = normal((2, 5), 204)
    want = vp.route_grad(x.cuda(), out["ids"], out["weights"], d.cuda(), score=score, renorm=renorm)
    d[0, 3:], d[1, 3], d[1, 4] = math.nan, math.inf, -math.inf
    got = vp.route_grad(x.cuda(), out["ids"], out["weights"], d.cuda(), score=score, renorm=renorm)
    assert torch.isfinite(want).all() and torch.equal(got, want)


# ------------------------------------------------------------------ merge

@pytest.mark.parametrize("T,k,H", [(1, 1, 8), (3, 2, 264), (7, 9, 72), (5, 17, 4104), (33, 8, 7168)])
@pytest.mark.parametrize("dtype", FLOATS, ids=str)
def test_the_gradient_of_a_weight_that_is_zero(vp, T, k, H, dtype):
    """<d_out, row> there too; 0 where the row of a dropped slot is no numbers."""
    rows, w, d = normal((T * k, H), 210, dtype), normal((T, k), 211), normal((T, H), 212, dtype)
    w[:, k - 1] = 0.0
    w[0, 0] = -0.0
    rows[k - 1, H - 1] = math.nan
    if T > 1:
        rows[2 * k - 1, 3] = math.inf
    _, gw = vp.merge_grad(d.cuda(), rows.cuda(), w.cuda())
    prod = d.double()[:, None, :] * rows.double().view(T, k, H)
    want, size = prod.sum(2), prod.abs().sum(2)
    dropped = (w == 0) & ~torch.isfinite(want)
    assert dropped[0, k - 1] and int(dropped.sum()) == min(T, 2)
    assert (gw.cpu()[dropped] == 0).all()
    near(gw.cpu()[~dropped], want[~dropped], (H + 2) * 2.0 ** -24 * size[~dropped], "d_weights")


def test_the_gradient_of_zero_weights_against_differences(vp):
    T, k, H = 2, 3, 16
    rows, d, w = normal((T * k, H), 213), normal((T, H), 214), torch.zeros(T, k)
    _, gw = vp.merge_grad(d.cuda(), rows.cuda(), w.cuda())
    f = lambda v: float((d.double() * vp.merge(rows.cuda(), v.cuda()).double().cpu()).sum())  # noqa: E731
    for i in range(T):
        for j in range(k):
            h = torch.zeros(T, k)
            h[i, j] = 0.5   # the merge is linear in its weights
            assert abs((f(h) - f(-h)) - float(gw[i, j])) < 1e-5


# ---------------------------------------------------------------- streams

def test_outputs_come_from_the_stream_they_are_written_on(vp):
    """Memory that the current stream freed, and may still be using, is not handed to a call on another stream."""
    T, k, H = 4096, 2, 4096
    rows, w = torch.ones((T * k, H), dtype=torch.bfloat16, device="cuda"), torch.ones((T, k), device="cuda")
    off = torch.tensor([0, 2 * T]).cuda()
    wt = torch.ones((1, 512, H), dtype=torch.bfloat16, device="cuda")
    logits = torch.zeros((1 << 20, 16), device="cuda")
    pre = torch.ones((T * k, H), dtype=torch.bfloat16, device="cuda")
    routing = torch.zeros((8, 1 << 20, 1), dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    r, q, qw = vp.route(logits, 2), vp.mx_quantize(rows), vp.mx_quantize(wt)
    calls = dict(
        merge=lambda s: vp.merge(rows, w, stream=s), merge_grad=lambda s: vp.merge_grad(rows[:T], rows, w, stream=s)[0],
        quantize=lambda s: vp.mx_quantize(rows, stream=s),
        dequantize=lambda s: vp.mx_dequantize(q, H, stream=s),
        matmul=lambda s: vp.expert_matmul(rows, wt, off, stream=s),
        grad_x=lambda s: vp.expert_matmul_grad_x(rows[:, :512], wt, off, stream=s),
        grad_w=lambda s: vp.expert_matmul_grad_w(rows, rows, off, stream=s),
        gate_grad=lambda s: vp.expert_gate_grad(pre[:, :H // 2], pre, off, stream=s),
        mx=lambda s: vp.expert_matmul_mx(q, qw, off, H, stream=s),
        route=lambda s: vp.route(logits, 2, stream=s)["weights"],
        route_grad=lambda s: vp.route_grad(logits, r["ids"], r["weights"], r["weights"], stream=s),
        demand=lambda s: vp.demand(routing, 8, 8, 64, stream=s)["sorted_tok"])
    for name, call in calls.items():
        torch.cuda.synchronize()
        like = call(None)
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        freed = [torch.empty_like(like) for _ in range(8)]
        places = {t.data_ptr() for t in freed}
        del freed
        side.wait_stream(torch.cuda.current_stream())
        got = call(side)
        side.synchronize()
        assert got.data_ptr() not in places, name
        assert torch.equal(got, like), name


# ---------------------------------------------------------------- offsets

BAD_OFFSETS = [[0, 10, 21], [0, 15, 10], [-3, 5, 20], [0, 2 ** 40, 2 ** 41], [5, 3, 20], [20, 0, 20], [0, -2 ** 63, 20],
               [-2 ** 63, 2 ** 63 - 1, 20]]


def test_the_gates_gradient_reports_offsets_out_of_order(vp):
    dh, pre = normal((20, 32), 220, torch.bfloat16).cuda(), normal((20, 64), 221, torch.bfloat16).cuda()
    for bad in BAD_OFFSETS + [[0, 5, 3, 20], [7, 0]]:
        st = vp.new_status()
        vp.expert_gate_grad(dh, pre, torch.tensor(bad).cuda(), status=st)
        assert vp.read_status(st) == vp.INVALID_ARGUMENT, bad


def test_products_of_offsets_out_of_order_write_nothing(vp):
    for R, N, K, L in ((20, 32, 64, 2), (2304, 2064, 264, 2), (8205, 2064, 64, 2)):
        x, w = normal((R, K), 222, torch.bfloat16).cuda(), normal((L, N, K), 223, torch.bfloat16).cuda()
        dy = normal((R, N), 224, torch.bfloat16).cuda()
        xq = wq = None
        if K % 32 == 0:
            xq, wq = vp.mx_quantize(x), vp.mx_quantize(w)
        for bad in BAD_OFFSETS + [[0, R, 0], [R, 0, R], [0, R + 1, R + 1], [1, 0, R]]:
            off = torch.tensor(bad).cuda()
            if all(0 <= a <= b <= R for a, b in zip(bad, bad[1:])):
                continue
            calls = [
                ((R, N), torch.bfloat16, lambda o, st: vp.expert_matmul(x, w, off, out=o, status=st)),
                ((R, N // 2), torch.bfloat16, lambda o, st: vp.expert_matmul(x, w, off, gated=True, out=o, status=st)),
                ((R, K), torch.bfloat16, lambda o, st: vp.expert_matmul_grad_x(dy, w, off, out=o, status=st)),
                ((L, N, K), torch.float32, lambda o, st: vp.expert_matmul_grad_w(dy, x, off, out=o, status=st))]
            if xq is not None:
                calls.append(((R, N), torch.bfloat16, lambda o, st: vp.expert_matmul_mx(xq, wq, off, K, out=o, status=st)))
            for shape, dtype, call in calls:
                st, out = vp.new_status(), torch.full(shape, 7.0, dtype=dtype, device="cuda")
                call(out, st)
                assert vp.read_status(st) == vp.INVALID_ARGUMENT, bad
                assert (out == 7.0).all(), bad


def test_errors_without_a_status_are_kept(vp):
    x, w = normal((20, 64), 225, torch.bfloat16).cuda(), normal((2, 32, 64), 226, torch.bfloat16).cuda()
    dy, pre = normal((20, 32), 227, torch.bfloat16).cuda(), normal((20, 64), 228, torch.bfloat16).cuda()
    off = torch.tensor([0, 15, 10]).cuda()
    ids = torch.tensor([[0, 1, 8]], dtype=torch.int32).cuda()
    one, counts = torch.ones(1, 3).cuda(), torch.full((2, 4), -1, dtype=torch.int32).cuda()
    xq, wq = vp.mx_quantize(x), vp.mx_quantize(w)
    vp.unclaimed_status()
    assert vp.unclaimed_status() == 0
    for call in (lambda: vp.expert_matmul(x, w, off), lambda: vp.expert_matmul_grad_x(dy, w, off),
                 lambda: vp.expert_matmul_grad_w(dy, x, off), lambda: vp.expert_gate_grad(dy, pre, off),
                 lambda: vp.expert_matmul_mx(xq, wq, off, 64), lambda: vp.expert_offsets(counts, 0),
                 lambda: vp.route_grad(torch.zeros(1, 8).cuda(), ids, one, one)):
        call()
        assert vp.unclaimed_status() == vp.INVALID_ARGUMENT
        assert vp.unclaimed_status() == 0   # taken
    st = vp.new_status()
    vp.expert_matmul(x, w, off, status=st)
    assert vp.unclaimed_status() == 0 and vp.read_status(st) == vp.INVALID_ARGUMENT
    with torch.cuda.stream(torch.cuda.Stream()):
        vp.expert_matmul(x, w, off)
        assert vp.unclaimed_status() == vp.INVALID_ARGUMENT


# ------------------------------------- more than 2^32 threads, wide strides

@pytest.fixture
def room():
    torch.cuda.empty_cache()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def ends(n, m=4097):
    """The first and last of n rows, and those around the 2^21st and the middle."""
    mid = [torch.arange(c - 3, c + 3) for c in (1 << 21, n // 2) if 3 < c < n - 3]
    return torch.cat([torch.arange(min(n, m)), *mid, torch.arange(n - min(n, m), n)]).unique().cuda()


def test_merge_of_two_to_the_26_tokens(vp, room):
    T, H = (1 << 26) + 5, 8   # 64 threads a token
    rows = torch.empty((T, H), dtype=torch.bfloat16, device="cuda").normal_()
    w = torch.full((T, 1), 0.5, device="cuda")
    assert torch.equal(vp.merge(rows, w), rows * 0.5)
    g, gw = vp.merge_grad(rows, rows, w)
    assert torch.equal(g, rows * 0.5)
    at = ends(T)
    near(gw[at, 0], (rows[at].double() ** 2).sum(1).cpu(), 2e-6 * (rows[at].double() ** 2).sum(1).cpu())
    assert (gw > 0).all()


def test_gate_gradient_of_two_to_the_24_rows(vp, room):
    R, I = (1 << 24) + 5, 8   # 256 threads a row
    pre = torch.empty((R, 2 * I), dtype=torch.bfloat16, device="cuda").normal_()
    dh = torch.empty((R, I), dtype=torch.bfloat16, device="cuda").normal_()
    st = vp.new_status()
    got = vp.expert_gate_grad(dh, pre, torch.tensor([0, R]).cuda(), status=st)
    assert vp.read_status(st) == 0
    at = ends(R)
    small = vp.expert_gate_grad(dh[at], pre[at], torch.tensor([0, len(at)]).cuda())
    assert torch.equal(got[at], small)


def test_four_bit_rows_two_to_the_24(vp, room):
    R, K = (1 << 24) + 5, 1056   # 256 threads a row
    x = torch.empty((R, K), dtype=torch.bfloat16, device="cuda")
    at = ends(R)
    x[at] = normal((len(at), K), 230, torch.bfloat16).cuda()
    want = vp.mx_quantize(x[at])
    q = vp.mx_quantize(x)
    assert torch.equal(q[at], want)
    del x
    assert torch.equal(vp.mx_dequantize(q, K)[at], vp.mx_dequantize(want, K))


def test_routes_of_two_to_the_28_tokens(vp, room):
    T = (1 << 28) + 5   # sixteen threads a token
    x = torch.empty((T, 2), dtype=torch.bfloat16, device="cuda").normal_()
    got = vp.route(x, 1, renorm=True)
    assert torch.equal(got["ids"][:, 0], (x[:, 1] > x[:, 0]).int()) and (got["weights"] == 1).all()


def test_route_gradient_of_two_to_the_26_tokens(vp, room):
    T = (1 << 26) + 5   # 64 threads a token
    x = torch.empty((T, 2), dtype=torch.bfloat16, device="cuda").normal_()
    d = torch.ones((T, 1), device="cuda")
    out = vp.route(x, 1, score="sigmoid", renorm=False)
    got = vp.route_grad(x, out["ids"], out["weights"], d, score="sigmoid", renorm=False)
    at = ends(T)
    small = vp.route_grad(x[at], out["ids"][at], out["weights"][at], d[at], score="sigmoid", renorm=False)
    assert torch.equal(got[at], small) and ((got != 0).sum(1) == 1).all()


def far_rows(n, m, dtype, seed):
    """A matrix whose rows lie more than 4 MiB apart."""
    wide = torch.full((n, (5 << 20) // dtype.itemsize), 255 if dtype == torch.uint8 else math.nan, dtype=dtype, device="cuda")
    wide[:, :m] = normal((n, m), seed, dtype).cuda()
    return wide[:, :m]


@pytest.mark.parametrize("dtype", FLOATS, ids=str)
def test_rows_more_than_4_mib_apart(vp, dtype):
    rows, res, w = far_rows(6, 72, dtype, 240), far_rows(3, 72, dtype, 241), normal((3, 2), 242).cuda()
    out = far_rows(3, 72, dtype, 243)
    near_rows, near_res = rows.contiguous(), res.contiguous()
    assert torch.equal(vp.merge(rows, w, residual=res, out=out), vp.merge(near_rows, w, residual=near_res))
    g, gw = vp.merge_grad(res, rows, w, d_rows=far_rows(6, 72, dtype, 244))
    g2, gw2 = vp.merge_grad(near_res, near_rows, w)
    assert torch.equal(g, g2) and torch.equal(gw, gw2)
    x = far_rows(4, 96, dtype, 245)
    q = far_rows(4, vp.mx_row_bytes(96), torch.uint8, 246)
    assert torch.equal(vp.mx_quantize(x, out=q), vp.mx_quantize(x.contiguous()))
    back = vp.mx_dequantize(q, 96, out=far_rows(4, 96, dtype, 247))
    assert torch.equal(back, vp.mx_dequantize(q.contiguous(), 96, dtype=dtype))
    if dtype != torch.float32:
        dh, pre, off = far_rows(4, 32, dtype, 248), far_rows(4, 64, dtype, 249), torch.tensor([0, 4]).cuda()
        got = vp.expert_gate_grad(dh, pre, off, out=far_rows(4, 64, dtype, 250))
        assert torch.equal(got, vp.expert_gate_grad(dh.contiguous(), pre.contiguous(), off))
