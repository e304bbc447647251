"""Every kernel of the dense products, at sizes that the library says select it: tiles of both sizes, alone on a CU and two
of them, one part of the contraction and several, contractions of one step and of many, more tiles than workgroups, edges
inside tiles; and the norm's and dropout's by the lengths of their rows."""
import math

import pytest
import torch

import dense_reference as ref
from layer_reference import rounded
from test_gpu_dense import guarded, near, near_rounded, normal, strided, vp  # noqa: F401

pytestmark = pytest.mark.gpu

# direction, R, N, K, kernel, parts: None where any number does
PRODUCTS = [
    ("forward", 1, 8, 8, "few_rows", 1), ("forward", 17, 72, 2056, "few_rows", None), ("forward", 128, 264, 4096, "few_rows", None), ("forward", 40, 520, 1000, "few_rows", 1),
    ("forward", 33, 16384, 512, "few_rows", 1),
    ("forward", 129, 8, 8, "tiles_alone", 1), ("forward", 130, 136, 64, "tiles_alone", 1), ("forward", 1000, 1032, 200, "tiles_alone", 1),
    ("forward", 140, 264, 4104, "tiles_alone", None), ("forward", 3000, 2056, 72, "tiles_128", 1), ("forward", 6100, 4104, 40, "tiles_128", 1),
    ("forward", 4090, 4088, 1032, "tiles_256", 1), ("forward", 8190, 4088, 520, "tiles_256", 1),
    ("grad_x", 1, 8, 8, "tiles_alone", 1), ("grad_x", 130, 72, 136, "tiles_alone", 1), ("grad_x", 96, 2056, 520, "tiles_alone", None),
    ("grad_x", 3000, 72, 2056, "tiles_128", 1), ("grad_x", 4090, 1032, 4088, "tiles_256", 1),
    ("grad_w", 1, 8, 8, "tiles_alone", 1), ("grad_w", 0, 136, 264, "tiles_alone", 1), ("grad_w", 65, 136, 264, "tiles_alone", 1),
    ("grad_w", 5000, 264, 136, "tiles_alone", None), ("grad_w", 72, 2056, 3000, "tiles_128", 1), ("grad_w", 9000, 1024, 1032, "tiles_128", None),
    ("grad_w", 1030, 4088, 4088, "tiles_256", 1),
]


def check(vp, direction, R, N, K, dtype, seed=0):  # noqa: F811
    """One product with all of its epilogue against 64 bits (on the GPU, which has them too)."""
    d = lambda t: None if t is None else t.cuda()  # noqa: E731
    x, w, dy = (d(normal(s, seed + i, dtype, std)) for i, (s, std) in enumerate((((R, K), 1.0), ((N, K), K ** -0.5), ((R, N), 1.0))))
    if direction == "forward":
        b, res = d(normal((N,), seed + 4)), d(normal((R, N), seed + 5, dtype))
        for act, wide in (("gelu", False), ("none", True)):
            r = res.float() if wide else res
            y, err, z, e = ref.linear(x, w, b, act, r)
            out, untouched = guarded((R, N), r.dtype)
            pre, same = guarded((R, N), dtype, 8)
            vp.linear(x, w, b, act=act, residual=r, out=out, pre=pre)
            assert_near(out, y, rounded(err, y, out.dtype))
            assert_near(pre, z, rounded(e, z, dtype))
            untouched()
            same()
            again = vp.linear(x, w, b, act=act, residual=r, dtype=r.dtype)
            assert torch.equal(out, again)
    elif direction == "grad_x":
        pre, res = d(normal((R, K), seed + 4, dtype, 2.0)), d(normal((R, K), seed + 5, dtype))
        for act, r in (("silu", res), ("none", None)):
            p = None if act == "none" else pre
            dx, e = ref.linear_grad_x(dy, w, act, p, r)
            out, untouched = guarded((R, K), dtype, 8)
            vp.linear_grad_x(dy, w, act=act, pre=p, residual=r, out=out)
            assert_near(out, dx, rounded(e, dx, dtype))
            untouched()
    else:
        dw, e = ref.linear_grad_w(dy, x)
        out, untouched = guarded((N, K), torch.float32)
        vp.linear_grad_w(dy, x, out=out)
        assert_near(out, dw, e + 1e-30)
        untouched()
        assert torch.equal(out, vp.linear_grad_w(dy, x))


def assert_near(got, want, bound):
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), "%d of %d, worst %.3g" % (int(bad.sum()), bad.numel(), float((got.double() - want).abs()[bad].max()))


@pytest.mark.parametrize("case", PRODUCTS, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
def test_every_kernel(vp, case, dtype):  # noqa: F811
    direction, R, N, K, kernel, parts = case
    kind, n = vp.linear_kernel(R, N, K, direction)
    assert kind == kernel and (n == parts if parts else n > 1)
    check(vp, direction, R, N, K, dtype)


@pytest.mark.parametrize("direction", ["forward", "grad_x", "grad_w"])
def test_sizes_around_the_tiles(vp, direction):  # noqa: F811
    """Rows, columns and contractions just below, at and above the tiles' sides and the steps."""
    for R, N, K in ((127, 120, 56), (128, 128, 64), (129, 136, 72), (255, 248, 120), (256, 256, 128), (257, 264, 136), (383, 384, 192),
                    (511, 504, 256), (64, 512, 320), (16, 1016, 504), (513, 64, 1000)):
        check(vp, direction, R, N, K, torch.bfloat16)


def test_strides_of_4_mib_and_of_16_bytes(vp):  # noqa: F811
    """The longest stride that products take, and rows as dense as they can be."""
    wide = torch.full((300, (4 << 20) // 2), math.nan, dtype=torch.bfloat16, device="cuda")
    x, w = normal((300, 72), 1, torch.bfloat16), normal((300, 72), 2, torch.bfloat16, 0.1)
    wide[:, :72], wide[:, 1024:1096] = x.cuda(), w.cuda()
    far_x, far_w, far_y = wide[:, :72], wide[:, 1024:1096], wide[:, 2048:2348 - 4]
    y, err, _, _ = ref.linear(x, w[:296])
    near_rounded(vp.linear(far_x, far_w[:296], out=far_y), y, err)
    assert wide[:, 2344].isnan().all() and wide[:, 2047].isnan().all()
    dy = normal((300, 296), 3, torch.bfloat16)
    far_y.copy_(dy)
    dx, e = ref.linear_grad_x(dy, w[:296])
    near_rounded(vp.linear_grad_x(far_y, far_w[:296]), dx, e)
    dw, e = ref.linear_grad_w(dy, x)
    near(vp.linear_grad_w(far_y, far_x), dw, e + 1e-30)
    # eight columns: rows of 16 bytes
    y, err, _, _ = ref.linear(x[:, :8].contiguous(), w[:8, :8].contiguous())
    near_rounded(vp.linear(x[:, :8].contiguous().cuda(), w[:8, :8].contiguous().cuda()), y, err)


def test_neighbours_of_views_do_not_enter_sums(vp):  # noqa: F811
    """Operands inside larger tensors of NaN on every side, at sizes of each kernel."""
    for direction, R, N, K in (("forward", 50, 72, 264), ("forward", 200, 136, 1032), ("forward", 3000, 2056, 72), ("grad_x", 200, 136, 72),
                               ("grad_w", 200, 136, 72), ("grad_w", 3000, 264, 136), ("forward", 4090, 4088, 392)):
        place = lambda r, c, s: inside(normal((r, c), s, torch.bfloat16, 0.2))  # noqa: E731
        x, w, dy = place(R, K, 1), place(N, K, 2), place(R, N, 3)
        if direction == "forward":
            got, want = vp.linear(x, w, inside(normal((1, N), 4))[0]), vp.linear(x.contiguous(), w.contiguous(), normal((N,), 4).cuda())
        elif direction == "grad_x":
            got, want = vp.linear_grad_x(dy, w), vp.linear_grad_x(dy.contiguous(), w.contiguous())
        else:
            got, want = vp.linear_grad_w(dy, x), vp.linear_grad_w(dy.contiguous(), x.contiguous())
        assert got.isfinite().all() and torch.equal(got, want), direction


def inside(t):
    wide = torch.full((t.shape[0] + 16, t.shape[1] + 32), math.nan, dtype=t.dtype, device="cuda")
    out = wide[8:-8, 16:-16]
    out.copy_(t)
    return out


def test_the_smallest_workspace_is_enough(vp):  # noqa: F811
    """Bytes behind the workspace stay, and what it held before does not matter."""
    for direction, R, N, K in (("forward", 96, 256, 7168), ("forward", 256, 512, 4096), ("grad_x", 96, 4096, 512), ("grad_w", 5000, 264, 136)):
        need = vp.linear_workspace_bytes(R, N, K, direction)
        assert need > 0
        room = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")   # NaN
        x, w, dy = (normal(s, i, torch.bfloat16, 0.3).cuda() for i, s in enumerate(((R, K), (N, K), (R, N))))
        call = {"forward": lambda ws: vp.linear(x, w, ws=ws), "grad_x": lambda ws: vp.linear_grad_x(dy, w, ws=ws),
                "grad_w": lambda ws: vp.linear_grad_w(dy, x, ws=ws)}[direction]
        assert torch.equal(call(room[:need]), call(None))
        assert (room[need:] == 255).all()
        with pytest.raises(ValueError):
            call(room[:need - 1])
    T, H = 1000, 264
    need = vp.layer_norm_grad_workspace_bytes(T, H)
    room = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    x, d = normal((T, H), 1).cuda(), normal((T, H), 2).cuda()
    st = torch.rand(T, 2, device="cuda")
    assert all(torch.equal(a, b) for a, b in zip(vp.layer_norm_grad(d, x, st, ws=room[:need]), vp.layer_norm_grad(d, x, st)))
    need_b = vp.linear_act_grad_workspace_bytes(T, H)
    assert need_b <= need and (room[need:] == 255).all()
    room.fill_(255)
    assert torch.equal(vp.linear_act_grad(d, ws=room[:need_b])[1], vp.linear_act_grad(d)[1]) and (room[need_b:] == 255).all()


def test_graphs_of_every_kernel_replay(vp):  # noqa: F811
    """Captured products of all kinds beside eager ones, several replays with new inputs."""
    sizes = [("forward", 96, 256, 7168), ("forward", 200, 136, 4104), ("forward", 3000, 2056, 72), ("forward", 4090, 4088, 392),
             ("grad_x", 96, 2056, 520), ("grad_x", 4090, 392, 4088), ("grad_w", 5000, 264, 136), ("grad_w", 392, 4088, 4088)]
    sets = [[normal(s, i, torch.bfloat16, 0.3).cuda() for i, s in enumerate(((R, K), (N, K), (R, N)))] for _, R, N, K in sizes]

    def run():
        out = []
        for (direction, *_), (x, w, dy) in zip(sizes, sets):
            out.append(vp.linear(x, w, act="silu") if direction == "forward" else vp.linear_grad_x(dy, w) if direction == "grad_x"
                       else vp.linear_grad_w(dy, x))
        return out
    run()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kept = run()
    for i in range(3):
        for s in sets:
            for t in s:
                t.copy_(t.roll(1 + i, 0))
        eager = run()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, eager))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=str)
def test_rows_of_every_length_class(vp, dtype):  # noqa: F811
    """Rows at the last and first length of each way a norm holds them: 16 lanes, a wavefront, workgroups of 1 to 16
    wavefronts with two or four pieces of a lane, and rows that are read again."""
    n = 16 // dtype.itemsize
    for pieces in (16, 32, 33, 128, 129, 256, 1024, 1025, 2048, 2049, 4096, 4097):
        for H in (pieces * n, pieces * n - n + 1):
            T = 5 if pieces < 1000 else 2
            x, w, b = normal((T, H), 1, dtype), normal((H,), 2, dtype, 0.2, 1.0), normal((H,), 3, dtype, 0.2)
            y, err, stats, _ = ref.norm(x, w, b, 1e-5, True)
            near_rounded(vp.layer_norm(x.cuda(), w.cuda(), b.cuda()), y, err, str(H))
            dy, stats = normal((T, H), 4, dtype), stats.float()
            dx, e_x, dw, e_w, db, e_b = ref.norm_grad(dy, x, stats, w, True)
            got = vp.layer_norm_grad(dy.cuda(), x.cuda(), stats.cuda(), w.cuda())
            near_rounded(got[0], dx, e_x, str(H))
            near(got[1], dw, e_w + 1e-30, str(H))
            near(got[2], db, e_b + 1e-30, str(H))
            mask, scale = ref.kept(T, H, 0.4, 3)
            want, e = ref.dropout(x, mask, scale)
            near_rounded(vp.dropout(x.cuda(), 0.4, 3), want, e)


def test_more_rows_than_workgroups_hold_at_once(vp):  # noqa: F811
    """Workgroups that go on to further rows, in every class of lengths, with a last turn that some of them sit out."""
    for H, T in ((64, 70001), (1024, 20003), (2048, 5003), (8192, 2051), (32768, 1030), (33000, 300)):
        x = torch.empty(T, H, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(H))
        d = x.roll(7, 0).roll(3, 1)
        at = torch.tensor([0, 1, T // 2, T - 2, T - 1], device="cuda")
        st = torch.empty(T, 2, device="cuda")
        y = vp.layer_norm(x, stats=st)
        some = torch.empty(5, 2, device="cuda")
        assert torch.equal(y[at], vp.layer_norm(x[at], stats=some)) and torch.equal(st[at], some)
        dx, dw, db = vp.layer_norm_grad(d, x, st)
        assert torch.equal(dx[at], vp.layer_norm_grad(d[at], x[at], st[at], params=False)[0])
        u = (x.double() - st[:, :1].double()) * st[:, 1:].double()
        assert_near(dw, (d.double() * u).sum(0), (T + 8) * ref.U * (d.double() * u).abs().sum(0))
        assert_near(db, d.double().sum(0), (T + 8) * ref.U * d.double().abs().sum(0))


@pytest.mark.parametrize("case", [("forward", 2, 8, 1 << 20), ("forward", 200, 8, 1 << 20), ("forward", 2, 1 << 20, 8), ("forward", 130, 1 << 20, 8),
                                  ("grad_x", 200, 1 << 20, 8), ("grad_x", 2, 8, 1 << 20), ("grad_w", 3, 1 << 20, 8), ("grad_w", 200, 8, 1 << 20)], ids=str)
def test_the_widest_products(vp, case):  # noqa: F811
    direction, R, N, K = case
    check(vp, direction, R, N, K, torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
def test_the_longest_rows(vp, dtype):  # noqa: F811
    """2^20 values, the limit, and one less; every call on rows."""
    for H in (1 << 20, (1 << 20) - 1):
        x, w, dy = normal((3, H), 1, dtype), normal((H,), 2, dtype, 0.2, 1.0), normal((3, H), 3, dtype)
        y, err, stats, _ = ref.norm(x, w, w, 1e-5, True)
        near_rounded(vp.layer_norm(x.cuda(), w.cuda(), w.cuda()), y, err)
        stats = stats.float()
        dx, e_x, dw, e_w, db, e_b = ref.norm_grad(dy, x, stats, w, True, x)
        got = vp.layer_norm_grad(dy.cuda(), x.cuda(), stats.cuda(), w.cuda(), residual=x.cuda())
        near_rounded(got[0], dx, e_x)
        near(got[1], dw, e_w + 1e-30)
        near(got[2], db, e_b + 1e-30)
        mask, scale = ref.kept(3, H, 0.1, 5, 6)
        want, e = ref.dropout(x, mask, scale, dy)
        near_rounded(vp.dropout(x.cuda(), 0.1, 5, step=torch.tensor([6]).cuda(), residual=dy.cuda()), want, e)
        d, e, db, e_b = ref.act_grad(dy, x, "gelu")
        got, got_b = vp.linear_act_grad(dy.cuda(), x.cuda(), act="gelu")
        near_rounded(got, d, e)
        near(got_b, db, e_b + 1e-30)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
def test_rows_more_than_4_mib_apart(vp, dtype):  # noqa: F811
    def far(T, H, seed):
        wide = torch.full((T, (5 << 20) // dtype.itemsize), math.nan, dtype=dtype, device="cuda")
        wide[:, 3:3 + H] = normal((T, H), seed, dtype).cuda()
        return wide[:, 3:3 + H]
    x, dy, res, st = far(6, 200, 1), far(6, 200, 2), far(6, 200, 3), torch.rand(6, 2, device="cuda")
    near_x, near_dy, near_res = x.contiguous(), dy.contiguous(), res.contiguous()
    out = far(6, 200, 4)
    assert torch.equal(vp.layer_norm(x, out=out), vp.layer_norm(near_x))
    assert all(torch.equal(a, b) for a, b in zip(vp.layer_norm_grad(dy, x, st, residual=res, d_x=out),
                                                 vp.layer_norm_grad(near_dy, near_x, st, residual=near_res)))
    assert torch.equal(vp.dropout(x, 0.3, 1, residual=res, out=out), vp.dropout(near_x, 0.3, 1, residual=near_res))
    got, want = vp.linear_act_grad(dy, x, act="silu", out=out), vp.linear_act_grad(near_dy, near_x, act="silu")
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
