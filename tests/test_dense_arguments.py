"""What the questions about dense products make of sizes that the calls refuse (no GPU)."""
import pytest


@pytest.fixture(scope="module")
def vp():
    import os
    import paper_2609_34340_amd as vp
    if not os.path.exists(vp.LIB_PATH):
        from paper_2609_34340_amd import build
        build.build()
    return vp


@pytest.mark.parametrize("direction", ["forward", "grad_x", "grad_w"])
def test_sizes_past_32_bits_have_no_kernel(vp, direction):
    """Whose low 32 (for rows 64) bits are sizes of a product."""
    assert vp.linear_kernel(96, 256, 7168, direction) and vp.linear_workspace_bytes(96, 256, 7168) > 0
    for sizes in ((96, (1 << 32) + 256, 7168), (96, 256, (1 << 32) + 7168), (96, 256 - (1 << 32), 7168), ((1 << 64) + 96, 256, 7168)):
        with pytest.raises(ValueError):
            vp.linear_kernel(*sizes, direction)
        assert vp.linear_workspace_bytes(*sizes, direction) == 0
