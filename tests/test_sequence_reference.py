"""The 64-bit reference of the operators over tokens: its gradients against differences, its pieces against the whole."""
import numpy as np
import pytest

import sequence_reference as ref


def _scan_inputs(rng, N, L, C, S, G, gate):
    r = rng.standard_normal
    return {"u": r((N, L, C)), "delta": r((N, L, C)), "A": -np.exp(r((C, S))), "B": r((N, L, G, S)), "C": r((N, L, G, S)),
            "D": r(C), "z": r((N, L, C)) if gate else None, "bias": r(C), "state": r((N, C, S))}


@pytest.mark.parametrize("gate,softplus_on", [(True, True), (False, True), (True, False)])
def test_scan_gradients_match_central_differences(gate, softplus_on):
    rng = np.random.default_rng(1)
    N, L, C, S, G = 2, 5, 4, 3, 2
    x = _scan_inputs(rng, N, L, C, S, G, gate)
    if not softplus_on:
        x["delta"] = np.abs(x["delta"]) * 0.3 + 0.1
        x["bias"] = np.abs(x["bias"]) * 0.1
    lengths = [5, 3]
    dout, dlast = rng.standard_normal((N, L, C)), rng.standard_normal((N, C, S))

    def value(v):
        y, last = ref.scan(softplus_on=softplus_on, lengths=lengths, **v)
        return (y * dout).sum() + (last * dlast).sum()

    grads = ref.scan_grad(dout, softplus_on=softplus_on, lengths=lengths, dlast=dlast, **x)
    names = {"u": "du", "delta": "ddelta", "A": "dA", "B": "dB", "C": "dC", "D": "dD", "bias": "ddelta_bias", "state": "dstate"}
    if gate:
        names["z"] = "dz"
    for k, name in names.items():
        way = rng.standard_normal(x[k].shape)
        e = 1e-6
        # central differences are off by e^2 times a third derivative and by 2^-53 / e: 1e-9 of values of order 10
        diff = (value({**x, k: x[k] + e * way}) - value({**x, k: x[k] - e * way})) / (2 * e)
        assert abs(diff - (grads[name] * way).sum()) < 1e-6, name


@pytest.mark.parametrize("F,silu_on", [(1, True), (4, True), (3, False)])
def test_causal_gradients_match_central_differences(F, silu_on):
    rng = np.random.default_rng(2)
    N, L, C = 3, 6, 2
    v = {"x": rng.standard_normal((N, L, C)), "filt": rng.standard_normal((C, F)), "bias": rng.standard_normal(C),
         "state": rng.standard_normal((N, F - 1, C))}
    lengths = [6, 2, 0]
    dout, dlast = rng.standard_normal((N, L, C)), rng.standard_normal((N, F - 1, C))

    def value(v):
        out, last, _, _ = ref.causal(silu_on=silu_on, lengths=lengths, **v)
        return (out * dout).sum() + (last * dlast).sum()

    grads = dict(zip(("x", "filt", "bias", "state"), ref.causal_grad(dout, silu_on=silu_on, lengths=lengths, dlast=dlast, **v)))
    for k, g in grads.items():
        way = rng.standard_normal(v[k].shape)
        e = 1e-6
        diff = (value({**v, k: v[k] + e * way}) - value({**v, k: v[k] - e * way})) / (2 * e)
        assert abs(diff - (g * way).sum()) < 1e-6, k


def test_a_sequence_in_two_pieces_is_the_sequence():
    rng = np.random.default_rng(3)
    x = _scan_inputs(rng, 2, 9, 4, 3, 2, True)
    whole, end = ref.scan(**x)
    cut = lambda lo, hi: {k: v[:, lo:hi] if k in ("u", "delta", "B", "C", "z") else v for k, v in x.items()}
    first, mid = ref.scan(**cut(0, 4))
    second, last = ref.scan(**{**cut(4, 9), "state": mid})
    assert np.allclose(np.concatenate([first, second], 1), whole, rtol=1e-12) and np.allclose(last, end, rtol=1e-12)
    f, b, c = rng.standard_normal((4, 4)), rng.standard_normal(4), x["u"]
    whole, end, _, _ = ref.causal(c, f, b)
    first, mid, _, _ = ref.causal(c[:, :2], f, b)
    second, last, _, _ = ref.causal(c[:, 2:], f, b, state=mid)
    assert np.allclose(np.concatenate([first, second], 1), whole, rtol=1e-12) and np.array_equal(last, end)
