"""Infinities and NaN in parameters of the operators over tokens: what has no terms of theirs is not touched by them."""
import numpy as np
import pytest
import torch

import paper_1705_10591_amd as dconv
import sequence_reference as ref
from test_causal_gpu import NAN, TYPES, _half_step, _np
from test_causal_gpu import _inputs as _causal_inputs

pytestmark = pytest.mark.gpu
INF = float("inf")


def _same(got, want, tol, what):
    got = _np(got)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    assert np.array_equal(np.isinf(got), np.isinf(want)) and np.array_equal(np.sign(got[np.isinf(got)]), np.sign(want[np.isinf(want)])), what
    ok = np.isfinite(want)
    assert np.all(np.abs(got[ok] - want[ok]) <= tol[ok]), what


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C,F", [(12, 4), (9, 3), (66, 8)])
def test_filters_that_are_not_finite(C, F, dtype):
    """dx is 0 behind a sequence's end whatever the filter holds, and a row of dx or dstate has terms of tokens that count alone."""
    dt, L = TYPES[dtype], 50
    lengths = [0, 1, 2, 8, 23, 50]
    N = len(lengths)
    x, w, b, st, dout, dlast = _causal_inputs(C, dt, N, L, C, F)
    w[0, 0], w[1, F - 1], w[2, 1], w[3, :] = INF, -INF, NAN, INF
    ln = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    got = dconv.dconv_causal_grad(dout, x, w, b, silu=False, state=st, lengths=ln, dstate_out=dlast)
    for n, v in enumerate(lengths):
        assert not got.dx[n, v:].any()                   # (a NaN counts as one that is not 0)
    args = (_np(dout), _np(x), _np(w), _np(b), False, _np(st), lengths, _np(dlast))
    with np.errstate(invalid="ignore"):
        want = ref.causal_grad(*args)
        # F products, their sum and the state's gradient; a rounding to the type
        tol = [ref.E24 * (2 * F + 16) * m for m in ref.causal_grad(*args, mag=True)]
    for k, name in ((0, "dx"), (3, "dstate")):
        finite = np.where(np.isfinite(want[k]), want[k], 0.0)
        _same(getattr(got, name), want[k], np.nan_to_num(tol[k], posinf=0.0) * 1.01 + _half_step(finite, dt), name)
    assert torch.equal(got.dstate[0], dlast[0])          # of a sequence without tokens


@pytest.mark.parametrize("lowest", [-INF, torch.finfo(torch.float32).min])
@pytest.mark.parametrize("L,C,S,G", [(40, 70, 16, 1), (130, 64, 5, 1), (300, 66, 16, 1), (400, 24, 4, 2), (200, 64, 20, 1)])
def test_decays_that_leave_nothing(L, C, S, G, lowest):
    """exp(d A) with the lowest A is 0 at every token, and no token does nothing: states, outputs and gradients of sequences that end
    inside a tile, a chunk or before their first token are those of an A of -1e30."""
    from test_scan_gpu import NAMES, _check_grads, _check_scan, _inputs
    lengths = [0, 1, 17, L - 5, L]
    x, st, dout, dlast = _inputs(L + C, torch.float32, len(lengths), L, C, S, G)
    ln = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    hit = torch.rand((C, S), generator=torch.Generator().manual_seed(L)).cuda() < 0.3
    hit[0], hit[1, 0] = True, False
    same = dict(x, A=torch.where(hit, -1e30, x["A"]))
    x["A"] = torch.where(hit, lowest, x["A"])
    last = torch.full_like(st, NAN)
    starts = dconv.scan_starts(len(lengths), L, C, S, G)
    out = dconv.dconv_scan(**x, state=st, lengths=ln, state_out=last, starts=starts)
    _check_scan(same, st, lengths, True, torch.float32, out, last)
    assert torch.equal(last[0], st[0])
    for kept in (None, starts):
        got = dconv.dconv_scan_grad(dout, **x, state=st, lengths=ln, dstate_out=dlast, starts=kept)
        _check_grads(same, st, dout, dlast, lengths, True, torch.float32, got)
        assert torch.equal(got.dstate[0], dlast[0])
    cache, one = st.clone(), {k: v if v is None or k in ("A", "D", "delta_bias") else v[:, 0] for k, v in x.items()}
    one["delta"] = torch.where(torch.arange(C, device="cuda") == 0, -1e4, one["delta"])      # a step of 0: the state stays
    one["delta_bias"] = None
    dconv.dconv_scan_step(**one, state=cache)
    assert torch.equal(cache[:, 0], st[:, 0]) and torch.isfinite(cache).all()
