"""What the layer calls make of their arguments before anything is enqueued (no GPU)."""
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


def test_the_kernel_that_sizes_select(vp):
    L = vp.lib()
    assert vp.expert_kernel(64, 4, 4096, 4096) == "few_rows" and vp.expert_kernel(32768, 4, 4096, 4096) == "tiles_256"
    assert vp.expert_kernel(64, 4, 4096, 4096, mode="grad_x") == "tiles_128"
    assert vp.expert_kernel(0, 1, 8, 8, mode="grad_w") == "tiles_128"
    assert vp.route_lanes(1, 256) == 64 and vp.route_lanes(16384, 256) == 16 and vp.route_lanes(16384, 257) == 64
    for args in ((3, 0, 0, 8, 1, 16, 32), (0, 2, 0, 8, 1, 16, 32), (0, 0, 2, 8, 1, 16, 32), (1, 1, 0, 8, 1, 16, 32),
                 (2, 0, 1, 8, 1, 16, 32), (0, 0, 0, -1, 1, 16, 32), (0, 0, 0, 8, 0, 16, 32), (0, 0, 0, 8, 1, 12, 32),
                 (0, 0, 1, 8, 1, 24, 32), (0, 1, 0, 8, 1, 16, 48), (0, 0, 0, 1 << 31, 1, 16, 32)):
        assert L.vp_expert_kernel(*args) < 0, args
    for args in ((-1, 8), (1, 0), (1, 4097)):
        assert L.vp_route_lanes(*args) < 0
    with pytest.raises(ValueError):
        vp.expert_kernel(8, 1, 12, 32)
    with pytest.raises(ValueError):
        vp.route_lanes(1, 4097)


def test_route_parameters_are_those_of_the_call(vp):
    from paper_2609_34340_amd.layer import _route_params
    scale, groups, renorm = torch.tensor(1.0), torch.tensor(2), torch.tensor(True)
    p = _route_params("softmax", 4, groups, None, 1, renorm, scale)._obj
    assert (p.scale, p.n_groups, p.top_groups, p.renorm) == (1.0, 2, 2, 1)
    scale.fill_(2.5)
    groups.fill_(4)
    renorm.fill_(False)
    p = _route_params("softmax", 4, groups, None, 1, renorm, scale)._obj
    assert (p.scale, p.n_groups, p.top_groups, p.renorm) == (2.5, 4, 4, 0)


def test_route_parameters_past_32_bits_are_refused(vp):
    from paper_2609_34340_amd.layer import _route_params
    for bad in (dict(n_groups=(1 << 32) + 1), dict(top_groups=1 << 31), dict(group_top=-(1 << 31)), dict(k=(1 << 32) + 4)):
        how = {**dict(score="softmax", k=4, n_groups=1, top_groups=1, group_top=1, renorm=True, scale=1.0), **bad}
        with pytest.raises(ValueError):
            _route_params(**how)


def test_taking_a_status_needs_a_place(vp):
    assert vp.lib().vp_take_status(None, None) == vp.INVALID_ARGUMENT


def test_tensors_of_another_device_are_refused(vp, monkeypatch):
    from types import SimpleNamespace as Plain
    from paper_2609_34340_amd.layer import _queue
    on = lambda i: Plain(get_device=lambda: i)  # noqa: E731
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    here, there = Plain(device_index=0, cuda_stream=7), Plain(device_index=1, cuda_stream=8)
    assert _queue(here, on(0), None, on(0)) == 7
    for args in ((None, on(0), on(1)), (None, on(1), on(1)), (here, on(1)), (there, on(0)), (there, on(1)), (None, on(0), on(-1))):
        with pytest.raises(ValueError):
            _queue(*args)
