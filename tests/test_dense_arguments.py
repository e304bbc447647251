"""What the questions about dense products answer: the kernels of few rows by wide outputs, and sizes that the calls refuse
(no GPU)."""
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


def test_wide_outputs_read_their_weights_once(vp):
    """From 65 rows on few_rows goes through the weights twice, and tiles do not; up to 32 rows it stays."""
    for R, N, K in ((65, 14336, 4096), (96, 28672, 4096), (128, 28672, 8192), (128, 131072, 4096), (65, 1 << 20, 2048)):
        assert vp.linear_kernel(R, N, K)[0] in ("tiles_alone", "tiles_128"), (R, N, K)
    for R, N, K in ((64, 131072, 4096), (48, 57344, 4096)):
        assert vp.linear_kernel(R, N, K) == ("tiles_128", 1), (R, N, K)
    for R, N, K in ((1, 28672, 4096), (32, 131072, 4096), (61, 4096, 4096), (96, 256, 7168), (128, 1024, 4096)):
        assert vp.linear_kernel(R, N, K)[0] == "few_rows", (R, N, K)
