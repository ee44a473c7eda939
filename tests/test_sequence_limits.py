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


@pytest.mark.gpu
@pytest.mark.parametrize("L,C,S", [(130, 70, 16), (400, 64, 4), (300, 24, 20)])
def test_workspaces_and_starts_aligned_to_16_bytes_and_no_more(L, C, S, monkeypatch):
    import torch
    from test_scan_gpu import _inputs
    x, st, dout, dlast = _inputs(L, torch.float32, 2, L, C, S, 1)
    starts = dconv.scan_starts(2, L, C, S)
    off = torch.empty(starts.numel() + 4, device="cuda")[4:]

    def calls(s):
        y = dconv.dconv_scan(**x, state=st, starts=s)
        return [y] + [t for k in (s, None) for t in dconv.dconv_scan_grad(dout, **x, state=st, dstate_out=dlast, starts=k)]

    want = calls(starts)
    monkeypatch.setattr(q, "_workspace", lambda n, like: like.new_empty((max(n, 16) + 3) // 4 + 4, dtype=torch.float32)[4:])
    got = calls(off)
    assert off.data_ptr() % 32 == 16
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("sizes", [(1 << 31, 4, 64, 16), (1, 1 << 31, 64, 16), (1, 4, 1 << 31, 16), (1, 4, 64, 1 << 40)])
def test_starts_of_sizes_beyond_32_bits_are_a_bad_shape(sizes):
    with pytest.raises(dconv.DconvError) as e:
        dconv.scan_starts(*sizes)
    assert e.value.status == SHAPE


@pytest.mark.gpu
def test_more_rows_than_32_bits_are_a_bad_shape():
    import torch
    many = lambda *s, t=torch.bfloat16: torch.zeros((1, *s), dtype=t, device="cuda").expand(1 << 31, *s)      # one row of memory
    w, A = torch.zeros((1, 4), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, 1), device="cuda")
    x, B = many(1, 1), many(1, 1, 1)
    for call in (lambda: dconv.dconv_causal(x, w), lambda: dconv.dconv_causal_grad(x, x, w), lambda: dconv.dconv_scan(x, x, A, B, B),
                 lambda: dconv.dconv_scan_grad(x, x, x, A, B, B)):
        with pytest.raises(dconv.DconvError) as e:
            call()
        assert e.value.status == SHAPE
