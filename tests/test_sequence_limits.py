"""Sizes at the limits that the operators over tokens document."""
import pytest

import paper_1705_10591_amd as dconv
from paper_1705_10591_amd import sequence as q
from test_sequence_abi import CAUSAL, SHAPE, _pack, causal


@pytest.mark.parametrize("C,F", [(1 << 28, 8), (1 << 28, 4), (215_000_000, 4), (1 << 30, 1)])
def test_filter_gradients_of_more_channels_than_a_launch_holds(C, F):
    """One token of so many channels fits the launch that makes dx, while dfilt and dbias have a value for every tap: the call is
    refused before either.  A launch holds 2^32 - 1 threads, four for each of the (F + 1) C values."""
    assert 4 * (F + 1) * C > (1 << 32) - 1
    sizes = {"dtype": 1, "N": 1, "L": 1, "C": C, "F": F}
    assert causal("dconv_causal_grad", **sizes) == SHAPE
    assert dconv.load_library().dconv_causal_workspace(_pack(CAUSAL, q._CAUSAL, sizes)) == -1


def test_filter_gradients_of_as_many_channels_as_a_launch_holds():
    C = ((1 << 32) - 256) // 4 // 5 // 64 * 64                      # of 4 taps
    need = dconv.load_library().dconv_causal_workspace(_pack(CAUSAL, q._CAUSAL, {"dtype": 1, "N": 1, "L": 1, "C": C, "F": 4}))
    assert need == 5 * C * 4
