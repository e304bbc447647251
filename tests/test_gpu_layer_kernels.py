"""Every kernel that the layer calls choose among, reached by sizes for which the library itself names it: the tiled
products of both sizes, several tiles to a workgroup, contractions of one step and of several, and the routers whose
tokens share a wavefront."""
import math

import pytest
import torch

import layer_reference as ref
from test_gpu_layer import check_route, cuts_of, near, normal, operands, strided

pytestmark = pytest.mark.gpu

HALVES = [torch.bfloat16, torch.float16]
FLOATS = HALVES + [torch.float32]
GX, GW = dict(mode="grad_x"), dict(mode="grad_w")


@pytest.fixture(scope="module")
def vp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_34340_amd as vp
    return vp


def shape(v):
    return str(v) if not isinstance(v, list) else "e%dr%d" % (len(v), sum(v))


# --------------------------------------------------------------- products

FORWARD = [
    # counts, N, K, kernel; 5 rows past the experts' come on top
    ([1025, 0, 700, 3, 571], 2064, 264, "tiles_128"),    # five steps; the last of eight bytes
    ([2048, 0, 700, 1349], 2064, 264, "tiles_128"),      # 561 tiles, 512 workgroups
    ([257, 1, 1037], 2064, 1032, "tiles_128"),
    ([4097, 0, 255, 1, 3847], 2064, 56, "tiles_256"),    # one step; 308 tiles, 256 workgroups
    ([2560, 1, 0, 2303, 340, 1], 2064, 328, "tiles_256"),
    ([64, 0, 700, 30], 528, 264, "few_rows"),
]


@pytest.mark.parametrize("counts,N,K,kernel", FORWARD, ids=shape)
@pytest.mark.parametrize("form", ["plain", "gated", "gated with pre"])
@pytest.mark.parametrize("dtype", HALVES, ids=str)
def test_forward(vp, counts, N, K, kernel, form, dtype):
    gated = form != "plain"
    if not gated:
        N -= 8   # no whole fragment at the end
    cuts, off, x, w = operands(counts, N, K, dtype, 5, 110)
    R, width = x.shape[0], N // 2 if gated else N
    assert vp.expert_kernel(R, len(counts), N, K, gated=gated) == kernel
    want, err = ref.product(torch.nan_to_num(x), w, cuts, gated)
    w = w.cuda()
    for xs in (x.cuda(), strided(x, 24)):
        out = torch.full((R, width + 16), 7.0, dtype=dtype).cuda()
        pre = torch.full((R, N + 8), 7.0, dtype=dtype).cuda() if form == "gated with pre" else None
        st = vp.new_status()
        y = vp.expert_matmul(xs, w, off, gated=gated, out=out[:, :width], pre=None if pre is None else pre[:, :N], status=st)
        assert vp.read_status(st) == 0
        near(y[:cuts[-1]], want[:cuts[-1]], ref.rounded(err, want, dtype)[:cuts[-1]], "y")
        assert (out[cuts[-1]:] == 7.0).all() and (out[:, width:] == 7.0).all()   # nothing else is written
        if pre is not None:
            z, ez = ref.product(torch.nan_to_num(x), w.cpu(), cuts)
            near(pre[:cuts[-1], :N], z[:cuts[-1]], ref.rounded(ez, z, dtype)[:cuts[-1]], "pre")
            assert (pre[cuts[-1]:] == 7.0).all() and (pre[:, N:] == 7.0).all()


BACKWARD = [
    # counts, N, K, kernel of grad x, kernel of grad w
    ([1025, 0, 700, 3, 571], 328, 1032, "tiles_128", "tiles_128"),
    ([2048, 0, 700, 1349], 56, 2064, "tiles_128", "tiles_128"),       # grad x: one step, 561 tiles for 512 workgroups
    ([4097, 0, 255, 1, 3847], 40, 2056, "tiles_256", "tiles_128"),    # one step, 308 tiles for 256 workgroups
    ([2560, 1, 0, 2303, 340, 1], 1288, 2056, "tiles_256", "tiles_256"),
]


@pytest.mark.parametrize("counts,N,K,kernel_x,kernel_w", BACKWARD, ids=shape)
@pytest.mark.parametrize("dtype", HALVES, ids=str)
def test_backward(vp, counts, N, K, kernel_x, kernel_w, dtype):
    cuts, off, x, w = operands(counts, N, K, dtype, 5, 120)
    R, L = x.shape[0], len(counts)
    assert vp.expert_kernel(R, L, N, K, **GX) == kernel_x and vp.expert_kernel(R, L, N, K, **GW) == kernel_w
    dy = torch.full((R, N), math.nan).to(dtype)
    dy[:cuts[-1]] = normal((cuts[-1], N), 122, dtype)
    want, err = ref.product(torch.nan_to_num(dy), w.transpose(1, 2), cuts)
    w, st = w.cuda(), vp.new_status()
    for pad in (0, 8):
        dys, xs = strided(dy, pad), strided(x, 3 * pad)
        out = torch.full((R, K + 8), 7.0, dtype=dtype).cuda()
        dx = vp.expert_matmul_grad_x(dys, w, off, out=out[:, :K], status=st)
        near(dx[:cuts[-1]], want[:cuts[-1]], ref.rounded(err, want, dtype)[:cuts[-1]], "dx")
        assert (out[cuts[-1]:] == 7.0).all() and (out[:, K:] == 7.0).all()
        dw = vp.expert_matmul_grad_w(dys, xs, off, status=st)
        assert vp.read_status(st) == 0
        for e in range(L):
            p, q = dy[cuts[e]:cuts[e + 1]].double(), x[cuts[e]:cuts[e + 1]].double()
            near(dw[e], p.t() @ q, (len(p) + 2) * 2.0 ** -24 * (p.abs().t() @ q.abs()), "dw of expert %d" % e)


MX = [
    ([4097, 0, 255, 1, 3847], 2064, 160, "tiles_256"),          # one step
    ([2560, 1, 0, 2303, 340, 1], 2064, 1056, "tiles_256"),      # five steps: four share a load of the powers
    ([1025, 0, 700, 3, 577], 2064, 1056, "tiles_128"),
    ([64, 0, 700, 30], 528, 1056, "few_rows"),
]


@pytest.mark.parametrize("counts,N,K,kernel", MX, ids=shape)
@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
@pytest.mark.parametrize("dtype", HALVES, ids=str)
def test_four_bit_blocks(vp, counts, N, K, kernel, gated, dtype):
    if not gated:
        N -= 8
    cuts, off = cuts_of(counts)
    R, L, width = cuts[-1] + 5, len(counts), N // 2 if gated else N
    assert vp.expert_kernel(R, L, N, K, gated=gated, mx=True) == kernel
    x = torch.full((R, K), math.nan)
    x[:cuts[-1]] = normal((cuts[-1], K), 130)
    # blocks of very different size: a power at a wrong place is seen
    x *= torch.exp2(torch.randint(-3, 4, (R, K // 32), generator=torch.Generator().manual_seed(131)).float()).repeat_interleave(32, 1)
    w = normal((L, N, K), 132, std=K ** -0.5)
    xq, wq = vp.mx_quantize(x.cuda()), vp.mx_quantize(w.cuda())
    dec = lambda q: ref.mx_decode(q.cpu().view(-1, q.shape[-1]), K)  # noqa: E731
    want, err = ref.product(torch.nan_to_num(dec(xq)), dec(wq).view(L, N, K), cuts, gated)
    wide = torch.full((R, xq.shape[1] + 112), 255, dtype=torch.uint8).cuda()
    wide[:, :xq.shape[1]] = xq
    for rows in (xq, wide[:, :xq.shape[1]]):
        out = torch.full((R, width + 8), 7.0, dtype=dtype).cuda()
        st = vp.new_status()
        y = vp.expert_matmul_mx(rows, wq, off, K, gated=gated, out=out[:, :width], status=st)
        assert vp.read_status(st) == 0
        near(y[:cuts[-1]], want[:cuts[-1]], ref.rounded(err, want, dtype)[:cuts[-1]], "y")
        assert (out[cuts[-1]:] == 7.0).all() and (out[:, width:] == 7.0).all()


@pytest.mark.parametrize("counts,N,K,kernel", [([1025, 0, 700, 3, 576], 2064, 264, "tiles_128"),
                                               ([2560, 1, 0, 2303, 341], 2064, 328, "tiles_256")], ids=shape)
def test_tiles_of_rows_4_mib_apart(vp, counts, N, K, kernel):
    """The longest stride the products take: rows up to 9 and 20 GiB into the buffer."""
    cuts, off, x, w = operands(counts, N, K, torch.bfloat16, 0, 145)
    R, L = x.shape[0], len(counts)
    assert vp.expert_kernel(R, L, N, K, gated=True) == vp.expert_kernel(R, L, N, K) == kernel
    far = torch.empty((R, 1 << 21), dtype=torch.bfloat16, device="cuda")
    far[:, :K], far[:, K:K + 8] = x.cuda(), math.nan
    far[:, 4096:4096 + 2 * N] = 7.0
    xs, ys, zs, w, st = far[:, :K], far[:, 4096:4096 + N], far[:, 4096 + N:4096 + 2 * N], w.cuda(), vp.new_status()
    x = x.cuda()
    assert torch.equal(vp.expert_matmul(xs, w, off, out=ys, status=st), vp.expert_matmul(x, w, off))
    pre = torch.empty((R, N), dtype=torch.bfloat16, device="cuda")
    y = vp.expert_matmul(xs, w, off, gated=True, out=ys[:, :N // 2], pre=zs, status=st)
    assert torch.equal(y, vp.expert_matmul(x, w, off, gated=True, pre=pre)) and torch.equal(zs, pre)
    assert torch.equal(vp.expert_matmul_grad_x(zs, w, off, out=far[:, 32768:32768 + K], status=st), vp.expert_matmul_grad_x(pre, w, off))
    assert torch.equal(vp.expert_matmul_grad_w(zs, xs, off, status=st), vp.expert_matmul_grad_w(pre, x, off))
    assert vp.read_status(st) == 0 and (far[:, 4096 + N // 2:4096 + N] == vp.expert_matmul(x, w, off)[:, N // 2:]).all()
    del far, xs, ys, zs, y
    torch.cuda.empty_cache()


def test_a_graph_of_tiled_products_replays(vp):
    """Several tiles to a workgroup, replayed with other work between: the results of the eager call, bit for bit."""
    counts, N, K = [4097, 0, 255, 1, 3847], 2064, 56
    cuts, off, x, w = operands(counts, N, K, torch.bfloat16, 5, 140)
    x, w, st = x.cuda(), w.cuda(), vp.new_status()
    assert vp.expert_kernel(x.shape[0], len(counts), N, K, gated=True) == "tiles_256"
    out = torch.zeros((x.shape[0], N // 2), dtype=torch.bfloat16, device="cuda")
    eager = vp.expert_matmul(x, w, off, gated=True, out=out, status=st).clone()
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        vp.expert_matmul(x, w, off, gated=True, out=out, status=st)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(g):
        vp.expert_matmul(x, w, off, gated=True, out=out, status=st)
    for _ in range(3):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
    assert vp.read_status(st) == 0


# ---------------------------------------------------------------- routing

ROUTES = [
    # T, E, k, score, bias, groups, kept, group_top, renorm, scale; sixteen lanes to a token, one token in the last block
    (2049, 7, 3, "softmax", True, 1, 1, 1, True, 1.0),
    (2049, 64, 8, "sigmoid", True, 8, 4, 2, True, 2.5),
    (2049, 65, 5, "softmax", False, 5, 3, 1, False, 1.0),
    (2049, 128, 8, "softmax", False, 1, 1, 1, True, 1.0),
    (4097, 129, 1, "sigmoid", False, 3, 1, 1, True, 1.0),
    (4097, 256, 8, "softmax", False, 1, 1, 1, False, 2.5),
    (4097, 256, 64, "sigmoid", True, 64, 33, 2, True, 1.0),
    # a wavefront to a token
    (2048, 128, 8, "softmax", False, 1, 1, 1, True, 1.0),
    (4096, 256, 8, "sigmoid", True, 8, 4, 2, True, 2.5),
]


@pytest.mark.parametrize("case", ROUTES, ids=lambda c: "-".join(map(str, c[:4])))
@pytest.mark.parametrize("dtype", FLOATS, ids=str)
def test_routes_of_many_tokens(vp, case, dtype):
    T, E, k, score, has_bias, groups, kept, top, renorm, scale = case
    assert vp.route_lanes(T, E) == (64 if T in (2048, 4096) else 16)
    x = normal((T, E), 150, std=2.0).to(dtype)
    x[5, 0:E:2] = -math.inf
    x[T - 1, E // 2:] = -math.inf
    x[T - 2] = -math.inf
    bias = 0.1 * normal((E,), 151) if has_bias else None
    how = dict(k=k, score=score, n_groups=groups, top_groups=kept, group_top=top, renorm=renorm, scale=scale)
    for logits in (x.cuda(), strided(x, 3)):
        got = vp.route(logits, bias=None if bias is None else bias.cuda(), **how)
        check_route(got, x, 1e-6, bias=bias, **how)
        assert (got["weights"][T - 2] == 0).all()


@pytest.mark.parametrize("E", [64, 128, 256])
@pytest.mark.parametrize("dtype", FLOATS, ids=str)
def test_ties_of_many_tokens_go_to_the_lowest_index(vp, E, dtype):
    T = 4100
    assert vp.route_lanes(T, E) == 16
    x = torch.zeros(T, E)
    x[1::4, E // 2:] = 1.0
    x[2::4, ::2] = -0.0
    x[3::4, 7] = x[3::4, E - 3] = 3.0
    for how in (dict(score="softmax"), dict(score="sigmoid", bias=torch.full((E,), 0.25).cuda()),
                dict(score="sigmoid", bias=torch.zeros(E).cuda(), n_groups=8, top_groups=3, group_top=2)):
        ids = vp.route(x.to(dtype).cuda(), 8, **how)["ids"].cpu().long()
        first, half = torch.arange(8), torch.arange(E // 2, E // 2 + 8)
        assert (ids[0::4] == first).all() and (ids[2::4] == first).all()
        assert (ids[3::4, :2] == torch.tensor([7, E - 3])).all()
        if "n_groups" not in how:
            assert (ids[1::4] == half).all() and (ids[3::4, 2:] == first[:6]).all()


@pytest.mark.parametrize("score,renorm", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_route_gradient_of_many_tokens(vp, score, renorm):
    T, E, k = 2051, 72, 6
    x, d = normal((T, E), 160, std=1.5), normal((T, k), 161)
    how = dict(score=score, renorm=renorm, scale=1.5)
    assert vp.route_lanes(T, E) == 16
    out = vp.route(x.cuda(), k, **how)
    got = vp.route_grad(x.cuda(), out["ids"], out["weights"], d.cuda(), **how)
    leaf = x.double().requires_grad_()
    w = ref.route_weights(leaf, out["ids"].cpu().long(), score, renorm, 1.5)
    (want,) = torch.autograd.grad((w * d.double()).sum(), leaf)
    row = (out["weights"].cpu().double() * d.double().abs()).sum(1, keepdim=True)
    near(got, want, ref.rounded(4e-6 * row.expand(T, E), want, torch.float32), "d_logits")
