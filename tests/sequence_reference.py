"""The operators over tokens in 64 bits, token by token, as their definitions read: what the tests compare with.

Every function takes numpy float64 arrays.  With `mag` it evaluates the same formulas on the absolute values of what is
multiplied and added: a result that is a sum of products of values, each of which has been rounded k times, is off by at
most k * 2^-24 * (the same sum of absolute values).  In the scan a term carries one decay for every token that it has come
through, so there `mag` is a number e by which every factor is enlarged as often as fp32 rounds it: the bound is
the result with e = 2^-24 minus that with e = 0.

Roundings of the scan's factors, in units of 2^-24 relative to them (a correctly rounded operation: 1; exp2, log2 and the
reciprocal, good to an ulp: 2):
  d     2 |raw| + 14: the argument of e^x is off by 2 |x| (the sum with the bias, the product with log2 e), the exponential 2,
        1 + e 1, the logarithm 2 and its constant 1, the quotient 5, products 3 (softplus' is at most its value over x)
  a     (that + 3) |d A| + 2, and 1 for the multiply-add that it enters; 72 |d A| more where a chunk adds up the d of
        its tokens (144 in the longest chunk here, so that a token's d is in 72 additions on average)
  silu  2 |z| + 8
"""
E24 = 2.0 ** -24

import numpy as np


def sigmoid(x):
    return 1.0 / (1.0 + np.exp(-x))


def silu(x):
    return x * sigmoid(x)


def dsilu(x):
    s = sigmoid(x)
    return s * (1.0 + x * (1.0 - s))


def softplus(x):
    return np.maximum(x, 0.0) + np.log1p(np.exp(-np.abs(x)))


def causal(x, filt, bias=None, silu_on=True, state=None, lengths=None):
    """-> out, state_out, s (before the activation), the sum of absolute terms of s."""
    N, L, C = x.shape
    F = filt.shape[1]
    out, s_all, mag = np.zeros_like(x), np.zeros_like(x), np.zeros_like(x)
    last = np.zeros((N, F - 1, C))
    b = np.zeros(C) if bias is None else bias
    for n in range(N):
        rows = np.zeros((F - 1 + L, C))
        if state is not None:
            rows[:F - 1] = state[n]
        ln = L if lengths is None else int(min(max(lengths[n], 0), L))
        rows[F - 1:F - 1 + ln] = x[n, :ln]
        for t in range(ln):
            s, m = b.copy(), np.abs(b)
            for j in range(F):
                s = s + filt[:, j] * rows[t + j]
                m = m + np.abs(filt[:, j] * rows[t + j])
            s_all[n, t], mag[n, t] = s, m
            out[n, t] = silu(s) if silu_on else s
        last[n] = rows[ln:ln + F - 1]
    return out, last, s_all, mag


def causal_grad(dout, x, filt, bias=None, silu_on=True, state=None, lengths=None, dlast=None, mag=False):
    """-> dx, dfilt, dbias, dstate"""
    N, L, C = x.shape
    F = filt.shape[1]
    _, _, s, s_mag = causal(x, filt, bias, silu_on, state, lengths)
    pos = np.abs if mag else (lambda v: v)
    w = pos(filt)
    dx, dfilt, dbias, dstate = np.zeros_like(x), np.zeros_like(filt), np.zeros(C), np.zeros((N, F - 1, C))
    for n in range(N):
        ln = L if lengths is None else int(min(max(lengths[n], 0), L))
        rows = np.zeros((F - 1 + L, C))
        if state is not None:
            rows[:F - 1] = state[n]
        rows[F - 1:F - 1 + ln] = x[n, :ln]
        drows = np.zeros((F - 1 + L, C))
        for t in range(ln):
            # (silu' may cancel: it is off by its second derivative, up to 1/2, times what s is off by)
            slope = (1.1 + 0.5 * s_mag[n, t] if mag else dsilu(s[n, t])) if silu_on else 1.0
            ds = pos(dout[n, t]) * slope
            for j in range(F):
                drows[t + j] += w[:, j] * ds
                dfilt[:, j] += ds * pos(rows[t + j])
            dbias += ds
        if dlast is not None:
            drows[ln:ln + F - 1] += pos(dlast[n])
        dx[n, :ln], dstate[n] = drows[F - 1:F - 1 + ln], drows[:F - 1]
    return dx, dfilt, dbias, dstate


def _per_channel(t, C):
    """[N, L, G, S] -> [N, L, C, S]"""
    return np.repeat(t, C // t.shape[2], axis=2)


def _steps(delta, bias, softplus_on, mag):
    """d, the factor of its derivative, and the roundings of d."""
    raw = delta + (0.0 if bias is None else bias)
    d = softplus(raw) if softplus_on else raw
    slope = sigmoid(raw) if softplus_on else np.ones_like(raw)
    k = 2 * np.abs(raw) + 14
    return (d, slope, k) if mag is None else (np.abs(d) * (1 + mag * k), slope * (1 + mag * k), k)


def _decay(d, A, k, mag):
    """exp(d A) of a token; enlarged with `mag`, where d is too."""
    if mag is None:
        return np.exp(d[:, None] * A)
    d = d / (1 + mag * k)
    x = d[:, None] * A
    return np.exp(x) * (1 + mag * ((k[:, None] + 75) * np.abs(x) + 3))


def _scan_states(u, d, A, B, state, lengths, k, mag):
    N, L, C = u.shape
    S = A.shape[1]
    h = np.zeros((N, L + 1, C, S))
    if state is not None:
        h[:, 0] = state
    Bc = _per_channel(B, C)
    for n in range(N):
        for t in range(L):
            if t < lengths[n]:
                h[n, t + 1] = _decay(d[n, t], A, k[n, t], mag) * h[n, t] + (d[n, t] * u[n, t])[:, None] * Bc[n, t] * (1 + 3 * (mag or 0))
            else:
                h[n, t + 1] = h[n, t]
    return h


def _lengths(lengths, N, L):
    return [L] * N if lengths is None else [int(min(max(v, 0), L)) for v in lengths]


def scan(u, delta, A, B, C, D=None, z=None, bias=None, softplus_on=True, state=None, lengths=None, mag=None):
    """-> out, state_out"""
    N, L, ch = u.shape
    ln = _lengths(lengths, N, L)
    pos = (lambda v: v) if mag is None else np.abs
    e = mag or 0.0
    d, _, k = _steps(delta, bias, softplus_on, mag)
    h = _scan_states(pos(u), d, A, pos(B), None if state is None else pos(state), ln, k, mag)
    y = (h[:, 1:] * pos(_per_channel(C, ch))).sum(-1)
    if D is not None:
        y = y + pos(D) * pos(u)
    y = y * (1 + e * (A.shape[1] + 4))
    if z is not None:
        y = y * pos(silu(z)) * (1 + e * (2 * np.abs(z) + 8))
    for n in range(N):
        y[n, ln[n]:] = 0.0
    return y, h[:, -1]


def scan_grad(dout, u, delta, A, B, C, D=None, z=None, bias=None, softplus_on=True, state=None, lengths=None, dlast=None,
              mag=None):
    """-> dict of the gradients"""
    N, L, ch = u.shape
    S, G = A.shape[1], B.shape[2]
    ln = _lengths(lengths, N, L)
    pos = (lambda v: v) if mag is None else np.abs
    e = mag or 0.0
    d, slope, k = _steps(delta, bias, softplus_on, mag)
    u, B, C, dout = pos(u), pos(B), pos(C), pos(dout)
    skip = np.zeros(ch) if D is None else pos(D)
    h = _scan_states(u, d, A, B, None if state is None else pos(state), ln, k, mag)
    Bc, Cc, Aw = _per_channel(B, ch), _per_channel(C, ch), pos(A)
    r = {"du": np.zeros_like(u), "ddelta": np.zeros_like(u), "dA": np.zeros_like(A), "dB": np.zeros_like(B),
         "dC": np.zeros_like(C), "dD": np.zeros(ch), "dz": np.zeros_like(u), "ddelta_bias": np.zeros(ch),
         "dstate": np.zeros((N, ch, S))}
    for n in range(N):
        g = np.zeros((ch, S)) if dlast is None else pos(dlast[n]).copy()
        for t in range(ln[n] - 1, -1, -1):
            dy = dout[n, t]
            if z is not None:
                y = (h[n, t + 1] * Cc[n, t]).sum(-1) + skip * u[n, t]
                # (silu' may cancel: its roundings are relative to 1)
                r["dz"][n, t] = dy * y * (dsilu(z[n, t]) if mag is None else 1 + np.abs(dsilu(z[n, t]))) * (1 + e * (2 * np.abs(z[n, t]) + 12 + S))
                dy = dy * pos(silu(z[n, t])) * (1 + e * (2 * np.abs(z[n, t]) + 9))
            a = _decay(d[n, t], A, k[n, t], mag)
            g = g + Cc[n, t] * dy[:, None]
            r["dC"][n, t] = (dy[:, None] * h[n, t + 1]).reshape(G, ch // G, S).sum(1)
            r["dB"][n, t] = (g * (d[n, t] * u[n, t])[:, None]).reshape(G, ch // G, S).sum(1)
            gb = (g * Bc[n, t]).sum(-1)
            ga = g * a * h[n, t]
            r["du"][n, t] = d[n, t] * gb + skip * dy
            dd = ((ga * Aw).sum(-1) + u[n, t] * gb) * slope[n, t]
            r["ddelta"][n, t] = dd
            r["ddelta_bias"] += dd
            r["dA"] += ga * d[n, t][:, None]
            r["dD"] += dy * u[n, t]
            g = g * a
        r["dstate"][n] = g
    # what the products and sums that lead to a gradient round: states, lanes and blocks of channels, all tokens
    for name, sums in (("du", S), ("ddelta", S), ("dB", ch // G), ("dC", ch // G), ("dA", N * L), ("dD", N * L), ("ddelta_bias", N * L + S)):
        r[name] *= 1 + e * (sums + 10)
    return r
