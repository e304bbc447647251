"""The layer example: routing, both exchanges, experts and merge of eight emulated ranks, against torch in 32 bits."""
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
def test_forward_and_backward(example, args):
    # bf16 rounds six times on the way (rows, pre, h, y, out, and as often back), each by at most 2^-8
    for name, err in example.main(args).items():
        assert err < 6 * 2.0 ** -8, (name, err)


def test_four_bit_rows(example):
    # values have at most 2 of 8 parts between levels: a quarter of their size at worst, far less on average
    errors = example.main(["--mx"])
    assert errors["weights"] < 0.25 and errors["out"] < 0.25
