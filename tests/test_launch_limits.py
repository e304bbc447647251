"""Calls whose rows would take more than 2^32 threads, a launch that runs in part and returns no error: packs are refused
before anything is enqueued, unpacks give a workgroup several rows."""
import pytest
import torch


@pytest.fixture(scope="module")
def vp():
    import os
    import paper_2609_34340_amd as vp
    if not os.path.exists(vp.LIB_PATH):
        from paper_2609_34340_amd import build
        build.build()
    return vp


P, BIG = 4096, 1 << 62   # an address and a workspace size that no refused call uses
LIMITS = [(16, 26), (2048, 26), (2064, 25), (4096, 25), (4112, 24), (8192, 24), (8208, 23), (14336, 23)]


@pytest.mark.parametrize("row,bits", LIMITS)
def test_packs_refuse_launches_of_2_to_the_32_threads(vp, row, bits):
    L, n = vp.lib(), 1 << bits
    pack = lambda T, k: L.vp_pack_rows(P, T, k, row, P, P, P, 0, 8, P, P, P, P, P, 8, P, 1 << 20, P, P, P, BIG, None)  # noqa: E731
    gather = lambda T, k: L.vp_pack_gather(P, row, T, k, P, P, 8, P, 1 << 20, P, P, BIG, None)  # noqa: E731
    for call in (pack, gather):
        assert call(n, 1) == call(n // 8, 8) == call(n - 7, 1) == vp.UNSUPPORTED


@pytest.mark.gpu
def test_unpack_of_two_to_the_26_rows(vp):
    """One source's rows of 16 bytes to one expert, 64 threads a row."""
    torch.cuda.empty_cache()
    R, row = (1 << 26) + 5, 16
    dev = dict(device="cuda")
    counts = torch.tensor([[0, 0], [R, 0]], dtype=torch.int32, **dev)
    sched = dict(K=torch.tensor([1], dtype=torch.int32, **dev), dst=torch.tensor([[1, 0]], dtype=torch.int32, **dev),
                 bytes=torch.tensor([[0, R * row]], dtype=torch.int64, **dev),
                 recv_src=torch.tensor([[1, 0]], dtype=torch.int32, **dev))
    recv = torch.zeros((R, vp.slot_bytes(row) // 8), dtype=torch.int64, **dev)
    recv[:, 0] = torch.arange(R, **dev)
    recv[:, 1] = ~recv[:, 0]
    out, st = torch.zeros_like(recv), vp.new_status()
    vp.unpack_rows(recv, row, counts, 0, sched, out, st)
    assert vp.read_status(st) == 0 and torch.equal(out, recv)
    del recv, out
    torch.cuda.empty_cache()
