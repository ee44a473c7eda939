"""Gradients that are sums over all tokens: how far their rounding errors may grow.

A sum of n terms of either sign that is added up one by one in 32 bits: the partial sum after k terms is about sqrt(k) terms, and
rounding it is off by 0.41 * 2^-24 of it (a uniform error of up to half a step, in the mean over a binade).  Altogether
0.41 * sqrt(n^2 / 2) terms, which is 0.29 * sqrt(n) * 2^-24 of the sum.  Sums of m such parts in 32 bits add 0.41 * sqrt(n m^2 / 2) terms,
0.29 * sqrt(m) of the sum, and each rounding of all parts on their way (to LDS, to memory, to the result) 0.41.  What is
added in 64 bits adds nothing.  The errors of a thousand sums and more have these sizes to a few hundredths: 1.2 times is allowed.
"""
import pytest
import torch

import paper_1705_10591_amd as dconv
from test_causal_gpu import TYPES
from test_causal_gpu import _inputs as _causal_inputs

pytestmark = pytest.mark.gpu


def _allowed(one_by_one, parts, roundings):
    return 1.2 * 2.0 ** -24 * (0.29 ** 2 * (one_by_one + (parts if parts > 1 else 0)) + 0.41 ** 2 * roundings) ** 0.5


def _off(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


# tokens that a thread adds up one by one, and how often it joins such sums: strips of 8, 128 in four parts, 128 in one
@pytest.mark.parametrize("dtype,N,L,C,F,tokens,parts", [("f32", 8, 250, 512, 4, 8, 1), ("f32", 3, 1021, 771, 4, 8, 1), ("f32", 8, 2048, 4096, 4, 32, 4),
                                                        ("f16", 64, 1000, 64, 3, 8, 1), ("f32", 8, 2048, 4096, 8, 128, 1)])
def test_gradients_of_filter_and_bias(dtype, N, L, C, F, tokens, parts):
    """Without the activation the terms are dout times x, which the multiply-adds do not round."""
    x, w, b, _, dout, _ = _causal_inputs(L, TYPES[dtype], N, L, C, F)
    got = dconv.dconv_causal_grad(dout, x, w, b, silu=False)
    want = torch.empty((C, F + 1), dtype=torch.float64, device="cuda")
    for lo in range(0, C, 256):
        s = slice(lo, lo + 256)
        d, rows = dout[:, :, s].double(), torch.nn.functional.pad(x[:, :, s].double(), (0, 0, F - 1, 0))
        for j in range(F):
            want[s, j] = (d * rows[:, j:j + L]).sum((0, 1))
        want[s, F] = d.sum((0, 1))
    # rounded on the way to LDS, to memory and to the result
    assert _off(got.dfilt, want[:, :F]) < _allowed(tokens, parts, 3)
    assert _off(got.dbias, want[:, F]) < _allowed(tokens, parts, 3)


def _allowed_of(terms, tiles):
    """Of the norm of the sums of `terms` [N, L, C] over tokens, as the scan's gradients add them up: a thread has every 16th token of a
    chunk, from the last to the first.  Terms of a gradient differ in size from token to token and are not independent, so that the
    partial sums are taken as they are instead of sqrt(k) terms: each is rounded to 0.41 * 2^-24 of itself, in the mean, and so is what
    goes to LDS, to memory and into the result."""
    N, L, C = terms.shape
    partial = terms.reshape(N, L // (16 * tiles), tiles, 16, C).flip(2).cumsum(2)
    chunk = partial[:, :, -1].sum(2)
    want = chunk.sum((0, 1))
    squares = sum(t.square().sum() for t in (partial, partial[:, :, -1], chunk, want))
    return 1.2 * 0.41 * 2.0 ** -24 * (squares.sqrt() / want.norm()).item(), want


# tiles whose tokens a thread adds up: chunks of 4, of 2 and of one sequence's 64
@pytest.mark.parametrize("N,L,C,G,tiles", [(4, 2048, 256, 1, 4), (8, 512, 192, 1, 2), (1, 1024, 512, 512, 64)])
def test_gradients_of_skip_and_step_bias(N, L, C, G, tiles):
    """Without a gate dD has terms of dout times u; the bias' gradient adds up ddelta, which is there to be compared with."""
    from test_scan_gpu import _inputs
    x, st, dout, dlast = _inputs(L + C, torch.float32, N, L, C, 16, G, gate=False)
    got = dconv.dconv_scan_grad(dout, **x, state=st, dstate_out=dlast)
    for name, terms in (("dD", dout.double() * x["u"].double()), ("ddelta_bias", got.ddelta.double())):
        tol, want = _allowed_of(terms, tiles)
        assert _off(getattr(got, name), want) < tol, name
