"""Packs and unpacks of more than 2^32 threads are refused before anything is enqueued (no GPU): such a launch runs in part
and returns no error."""
import pytest


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
def test_pack_and_unpack_refuse_launches_of_2_to_the_32_threads(vp, row, bits):
    L, n, slot = vp.lib(), 1 << bits, vp.slot_bytes(row)
    pack = lambda T, k: L.vp_pack_rows(P, T, k, row, P, P, P, 0, 8, P, P, P, P, P, 8, P, 1 << 20, P, P, P, BIG, None)  # noqa: E731
    gather = lambda T, k: L.vp_pack_gather(P, row, T, k, P, P, 8, P, 1 << 20, P, P, BIG, None)  # noqa: E731
    for call in (pack, gather):
        assert call(n, 1) == call(n // 8, 8) == call(n - 7, 1) == vp.UNSUPPORTED
    assert L.vp_unpack_rows(P, (n - 7) * slot, row, P, 8, 0, 8, P, P, P, P, 8, P, 1 << 20, P, P, BIG, None) == vp.UNSUPPORTED
    assert L.vp_pack_combine(P, 1 << 20, row, P, 8, 0, 8, P, P, P, 8, P, (n - 7) * row, P, P, P, BIG, None) == vp.UNSUPPORTED
    assert L.vp_unpack_combine(P, (n - 7) * slot, row, 8, 1, P, P, P, 0, 8, P, P, P, P, 8, P, P, P, BIG, None) == vp.UNSUPPORTED
