"""The causal convolution over tokens against its 64-bit definition: prompts, gradients, single tokens."""
import numpy as np
import pytest
import torch

import paper_1705_10591_amd as dconv
import sequence_reference as ref

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
NAN = float("nan")


def _half_step(t, dtype):
    """Rounding a value to its type: half a step, or of a subnormal number half of the smallest."""
    f = torch.finfo(dtype)
    return np.abs(t) * (f.eps / 2) + f.smallest_normal * f.eps / 2


def _np(t):
    return t.detach().double().cpu().numpy()


def _inputs(seed, dtype, N, L, C, F, pad=0):
    """Values of the type, x a slice of rows `pad` channels wider."""
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g).to(dtype)
    wide = r(N, L, C + pad).cuda()
    return wide[:, :, pad:], (0.5 * r(C, F)).to(dtype).cuda(), r(C).cuda(), r(N, F - 1, C).cuda(), r(N, L, C).cuda(), r(N, F - 1, C).cuda()


def _check(got, want, bound, dtype, what, floor=0.0):
    got = _np(got)
    assert np.all(np.isfinite(got)), what
    err = np.abs(got - want)
    tol = _half_step(want, dtype) + bound * (1 + torch.finfo(dtype).eps) + floor
    assert np.all(err <= tol), f"{what}: off by up to {np.max(err / tol):.3g} of the bound at {np.unravel_index(np.argmax(err - tol), err.shape)}"


def _out_bound(out, s, mag, F, silu):
    # s: F multiply-adds of a sum; silu: its slope is at most 1.1, and the exponential's argument is off by 2 |s|, the
    # exponential, the sum, the reciprocal and the product by 6 in all
    return ref.E24 * (1.1 * (F + 1) * mag + (2 * np.abs(s) + 8) * np.abs(out)) if silu else ref.E24 * (F + 1) * mag


SHAPES = [(1, 1, 1, 1), (1, 1, 64, 4), (2, 2, 8, 4), (3, 3, 9, 8), (2, 7, 67, 3), (1, 8, 512, 2), (4, 9, 100, 5), (2, 65, 130, 6),
          (1, 33, 2049, 7), (3, 200, 24, 4), (1, 1000, 16, 8)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,L,C,F", SHAPES)
def test_prompts(N, L, C, F, dtype):
    dt = TYPES[dtype]
    for k, (silu, bias, state, pad) in enumerate([(True, True, False, 0), (False, False, True, 3), (True, True, True, 8)]):
        x, w, b, st, _, _ = _inputs(10 * N + L + k, dt, N, L, C, F, pad)
        b, st = b if bias else None, st if state else None
        last = torch.full((N, F - 1, C), NAN, device="cuda", dtype=dt)
        out = torch.full((N, L, C + 2), NAN, device="cuda", dtype=dt)
        got = dconv.dconv_causal(x, w, b, silu=silu, state=st, out=out[:, :, 1:-1], state_out=last)
        assert got.data_ptr() == out[:, :, 1:-1].data_ptr()
        want, wlast, s, mag = ref.causal(_np(x), _np(w), None if b is None else _np(b), silu, None if st is None else _np(st))
        _check(got, want, _out_bound(want, s, mag, F, silu), dt, "out")
        assert np.array_equal(_np(last), wlast)
        assert torch.isnan(out[:, :, 0]).all() and torch.isnan(out[:, :, -1]).all()      # the columns beside are not touched


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C,F", [(70, 4), (8, 8), (513, 3)])
def test_padded_batches(C, F, dtype):
    """Lengths at both ends, inside a strip, on its border, out of range; what lies behind is NaN."""
    dt, L = TYPES[dtype], 70
    lengths = [0, 1, 2, 7, 8, 9, 32, 64, 69, 70, -3, 99]
    N = len(lengths)
    x, w, b, st, dout, dlast = _inputs(C, dt, N, L, C, F)
    for n, v in enumerate(lengths):
        x[n, min(max(v, 0), L):] = NAN
        dout[n, min(max(v, 0), L):] = NAN
    ln = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    want, wlast, s, mag = ref.causal(_np(x), _np(w), _np(b), True, _np(st), lengths)
    keep = st.clone()
    out = dconv.dconv_causal(x, w, b, state=st, lengths=ln, state_out=st)                 # over the state that it reads
    _check(out, want, _out_bound(want, s, mag, F, True), dt, "out")
    assert np.array_equal(_np(st), wlast)
    _check_grads(dout, x, w, b, keep, ln, lengths, dlast, True, dt)


def _check_grads(dout, x, w, b, st, ln, lengths, dlast, silu, dt):
    N, L, C = x.shape
    F = w.shape[1]
    got = dconv.dconv_causal_grad(dout, x, w, b, silu=silu, state=st, lengths=ln, dstate_out=dlast)
    opt = lambda t: None if t is None else _np(t)
    args = (_np(dout), _np(x), _np(w), opt(b), silu, opt(st), lengths, opt(dlast))
    want, mag = ref.causal_grad(*args), ref.causal_grad(*args, mag=True)
    # ds: s is off by F + 1, silu' by 12 beside; dx: F products and the state's gradient; sums over all tokens
    k = ref.E24 * np.array([2 * F + 16, F + 16 + N * L, F + 16 + N * L, 2 * F + 16])
    _check(got.dx, want[0], k[0] * mag[0], dt, "dx")
    _check(got.dfilt, want[1], k[1] * mag[1], torch.float32, "dfilt")
    _check(got.dbias, want[2], k[2] * mag[2], torch.float32, "dbias")
    if st is None:
        assert got.dstate is None
    else:
        _check(got.dstate, want[3], k[3] * mag[3], dt, "dstate")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,L,C,F", SHAPES)
def test_gradients(N, L, C, F, dtype):
    dt = TYPES[dtype]
    for k, (silu, bias, state, pad) in enumerate([(True, True, False, 0), (False, False, True, 3), (True, True, True, 8)]):
        x, w, b, st, dout, dlast = _inputs(20 * N + L + k, dt, N, L, C, F, pad)
        _check_grads(dout, x, w, b if bias else None, st if state else None, None, None, dlast if state and k == 2 else None, silu, dt)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,C,F", [(1, 1, 4), (1, 64, 1), (5, 67, 4), (3, 2050, 8), (300, 24, 2)])
def test_steps(N, C, F, dtype):
    """Tokens one at a time are the prompt; slots in any order, padding rows, a slot that is named twice."""
    dt, M = TYPES[dtype], N + 3
    x, w, b, _, _, _ = _inputs(N + C, dt, N, 3, C, F)
    cache = torch.randn((M, F - 1, C), generator=torch.Generator().manual_seed(5)).to(dt).cuda()
    slots = torch.randperm(M, generator=torch.Generator().manual_seed(6))[:N].to(torch.int32)
    for bad, at in ((-1, 1), (M, 2), (2147483647, 4), (-2147483648, N - 1)):
        if N > 4:
            slots[at] = bad
    if N > 4:
        slots[3] = slots[0]
    live = [n for n in range(N) if 0 <= slots[n] < M and slots[n] not in slots[:n]]
    before = cache.clone()
    start = torch.zeros((N, F - 1, C), dtype=dt, device="cuda")
    for n in live:
        start[n] = cache[slots[n]]
    lengths = torch.tensor([3 if n in live else 0 for n in range(N)], dtype=torch.int32, device="cuda")
    last = torch.empty_like(start)
    whole = dconv.dconv_causal(x, w, b, state=start, lengths=lengths, state_out=last)
    for t in range(3):
        out = torch.full((N, C), NAN, dtype=dt, device="cuda")
        dconv.dconv_causal_step(x[:, t], cache, w, b, slots=slots.cuda(), out=out)
        assert torch.equal(out, whole[:, t]), t          # the same operations in the same order
    for n in live:
        assert torch.equal(cache[slots[n]], last[n])
        before[slots[n]] = last[n]
    assert torch.equal(cache, before)                    # no other window changed
    plain = start.clone()
    assert torch.equal(dconv.dconv_causal_step(x[:, 0], plain, w, b)[live], whole[live, 0])


def test_a_sequence_without_tokens_adds_nothing_whatever_its_state_holds():
    N, L, C, F = 2, 20, 16, 4
    x, w, b, st, dout, dlast = _inputs(7, torch.float32, N, L, C, F)
    lengths = torch.tensor([20, 0], dtype=torch.int32, device="cuda")
    st[1], x[1], dout[1] = NAN, NAN, NAN
    got = dconv.dconv_causal_grad(dout, x, w, b, state=st, lengths=lengths, dstate_out=dlast)
    one = dconv.dconv_causal_grad(dout[:1], x[:1], w, b, state=st[:1], dstate_out=dlast[:1])
    assert torch.equal(got.dfilt, one.dfilt) and torch.equal(got.dbias, one.dbias)
    assert torch.equal(got.dx[0], one.dx[0]) and not got.dx[1].any() and torch.equal(got.dstate[1], dlast[1])


def test_rows_beyond_32_bits():
    """Tokens whose elements lie more than 2^31 (and 2^32 bytes) from the first."""
    N, L, C, F = 2, 3, 64, 4
    big = torch.empty(((1 << 31) + 4096,), dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(big, (N, L, C), ((1 << 31) - 100, 700, 1))
    out = torch.as_strided(big, (N, L, C), ((1 << 31) - 100, 700, 1), 350)
    small, w, b, _, _, _ = _inputs(1, torch.bfloat16, N, L, C, F)
    x.copy_(small)
    assert torch.equal(dconv.dconv_causal(x, w, b, out=out), dconv.dconv_causal(small, w, b))
    assert torch.equal(dconv.dconv_causal_grad(out, x, w, b).dx, dconv.dconv_causal_grad(out.contiguous(), small, w, b).dx)


def test_non_finite_values_stay_in_their_window():
    N, L, C, F = 1, 40, 16, 4
    x, w, b, _, dout, _ = _inputs(3, torch.float32, N, L, C, F)
    clean = dconv.dconv_causal(x, w, b)
    x[0, 17, 5] = float("inf")
    out = dconv.dconv_causal(x, w, b)
    hit = torch.zeros((N, L, C), dtype=torch.bool, device="cuda")
    hit[0, 17:21, 5] = True
    assert torch.equal(out[~hit], clean[~hit])
    assert not torch.equal(out[hit], clean[hit])


def test_captured_calls_replay():
    x, w, b, st, dout, dlast = _inputs(4, torch.bfloat16, 2, 50, 72, 4)
    cache = st.clone()

    def calls(out, last):
        dconv.dconv_causal(x, w, b, state=st, out=out, state_out=last)
        dconv.dconv_causal_step(x[:, 0], cache, w, b)
        return dconv.dconv_causal_grad(dout, x, w, b, state=st, dstate_out=dlast)

    out, last = torch.empty_like(x), torch.empty_like(st)
    eager = calls(out, last)
    want, wlast, moved = out.clone(), last.clone(), cache.clone()
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        grads = calls(out, last)
    for rep in range(3):
        out.fill_(NAN), last.fill_(NAN), cache.copy_(st)
        for t in grads:
            t.fill_(NAN)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(last, wlast) and torch.equal(cache, moved)
        assert all(torch.equal(a, e) for a, e in zip(grads, eager)), rep
        other = dconv.dconv_causal_grad(dout, x, w, b, state=st, dstate_out=dlast)       # eager work of its own workspace
        torch.cuda.synchronize()
        assert all(torch.equal(a, e) for a, e in zip(other, eager))
