"""The layer example inside its block: norm, router, shared expert, both exchanges, experts, merge and dropout, against torch
in 32 bits."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("moe_layer", os.path.join(ROOT, "examples", "moe_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("args", [[], ["--tokens", "33", "--hidden", "264", "--inner", "72", "--experts", "16", "--top-k", "4"],
                                  ["--tokens", "1", "--hidden", "64", "--inner", "64"]], ids=str)
def test_block_forward_and_backward(example, args):
    # bf16 rounds nine times on the longest way (norm, rows, pre, h, y, merge, out, and back through the same), each by at
    # most 2^-8 of a value's size
    errors = example.main(["--block"] + args)
    assert len(errors) == 10
    for name, err in errors.items():
        assert err < 9 * 2.0 ** -8, (name, err)
