"""The selective scan against its 64-bit definition: prompts, gradients, single tokens, and both operators in a row."""
import numpy as np
import pytest
import torch

import paper_1705_10591_amd as dconv
import sequence_reference as ref
from test_causal_gpu import TYPES, NAN, _check, _np

pytestmark = pytest.mark.gpu
NAMES = ("du", "ddelta", "dA", "dB", "dC", "dD", "dz", "ddelta_bias", "dstate")


def _inputs(seed, dtype, N, L, C, S, G, gate=True, skip=True, bias=True, state=True, softplus=True):
    """u and z are halves of one tensor, B and C columns of another; d is up to about 2, decays between e^-8 and 1."""
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g)
    rows = r(N, L, 2 * C).to(dtype).cuda()
    bc = r(N, L, 2 * G * S + 1).to(dtype).cuda()
    delta = (0.5 * r(N, L, C) if softplus else torch.rand((N, L, C), generator=g) * 0.2).to(dtype).cuda()
    x = {"u": rows[:, :, :C], "delta": delta, "A": -(torch.rand((C, S), generator=g) * 4).cuda(),
         "B": bc[:, :, 1:G * S + 1].unflatten(2, (G, S)), "C": bc[:, :, G * S + 1:].unflatten(2, (G, S)),
         "D": r(C).cuda() if skip else None, "z": rows[:, :, C:] if gate else None,
         "delta_bias": (r(C) - 1 if softplus else torch.rand(C, generator=g) * 0.1).cuda() if bias else None}
    st = r(N, C, S).cuda() if state else None
    return x, st, r(N, L, C).to(dtype).cuda(), r(N, C, S).cuda()


def _reference(x):
    v = {k: None if t is None else _np(t) for k, t in x.items()}
    v["bias"] = v.pop("delta_bias")
    return v


def _check_scan(x, st, lengths, softplus, dt, out, last, floor=0.0):
    v = _reference(x)
    opts = {"softplus_on": softplus, "state": None if st is None else _np(st), "lengths": lengths}
    want, lo, hi = (ref.scan(**v, **opts, mag=m) for m in (None, 0.0, ref.E24))
    _check(out, want[0], hi[0] - lo[0], dt, "out", floor)
    if last is not None:
        _check(last, want[1], hi[1] - lo[1], torch.float32, "state_out")


def _check_grads(x, st, dout, dlast, lengths, softplus, dt, got, floor=0.0):
    v = _reference(x)
    opts = {"softplus_on": softplus, "state": None if st is None else _np(st), "lengths": lengths,
            "dlast": None if dlast is None else _np(dlast)}
    want, lo, hi = (ref.scan_grad(_np(dout), **v, **opts, mag=m) for m in (None, 0.0, ref.E24))
    missing = {"dD": "D", "dz": "z", "ddelta_bias": "delta_bias"}
    for name in NAMES:
        t = getattr(got, name)
        if (name in missing and x[missing[name]] is None) or (name == "dstate" and st is None):
            assert t is None
            continue
        _check(t, want[name], hi[name] - lo[name], dt if name in ("du", "ddelta", "dB", "dC", "dz") else torch.float32, name, floor)


# (sequences, tokens, channels, states, groups); the last ones have chunks
SHAPES = [(1, 1, 1, 1, 1), (1, 2, 64, 16, 1), (2, 15, 65, 16, 1), (3, 16, 63, 5, 1), (1, 17, 130, 8, 2), (2, 33, 96, 32, 3),
          (2, 40, 70, 4, 1), (1, 64, 6, 3, 2), (1, 300, 64, 16, 1), (2, 1000, 20, 12, 1), (1, 513, 24, 20, 2)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,L,C,S,G", SHAPES)
def test_prompts_and_gradients(N, L, C, S, G, dtype):
    dt = TYPES[dtype]
    for k, opts in enumerate([{}, {"gate": False, "skip": False, "bias": False, "state": False}, {"softplus": False, "gate": False}]):
        if k and dtype == "f16":
            continue
        softplus = opts.get("softplus", True)
        x, st, dout, dlast = _inputs(N + L + C + k, dt, N, L, C, S, G, **opts)
        last = torch.full((N, C, S), NAN, device="cuda")
        wide = torch.full((N, L, C + 2), NAN, device="cuda", dtype=dt)
        starts = dconv.scan_starts(N, L, C, S, G)
        out = dconv.dconv_scan(**x, softplus=softplus, state=st, out=wide[:, :, 1:-1], state_out=last, starts=starts)
        _check_scan(x, st, None, softplus, dt, out, last)
        assert torch.isnan(wide[:, :, 0]).all() and torch.isnan(wide[:, :, -1]).all()
        dlast = None if k == 1 else dlast
        got = dconv.dconv_scan_grad(dout, **x, softplus=softplus, state=st, dstate_out=dlast, starts=starts)
        _check_grads(x, st, dout, dlast, None, softplus, dt, got)
        # states made again, chunk by chunk where there are chunks
        again = dconv.dconv_scan_grad(dout, **x, softplus=softplus, state=st, dstate_out=dlast)
        _check_grads(x, st, dout, dlast, None, softplus, dt, again)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("L,C,S,G", [(40, 70, 16, 1), (400, 66, 6, 2)])
def test_padded_batches(L, C, S, G, dtype):
    """Lengths at both ends, inside a tile, on its border and a chunk's, out of range; what lies behind is NaN."""
    dt = TYPES[dtype]
    lengths = [0, 1, 15, 16, 17, L - 1, L, -5, L + 7] + ([128, 144, 200, 257, 272] if L > 300 else [])
    N = len(lengths)
    x, st, dout, dlast = _inputs(L, dt, N, L, C, S, G)
    for n, v in enumerate(lengths):
        v = min(max(v, 0), L)
        for t in (x["u"], x["delta"], x["z"], x["B"], x["C"], dout):
            t[n, v:] = NAN
    ln = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    for t in x:
        if x[t] is not None and x[t].dim() > 2 and t != "A":
            assert torch.isnan(x[t]).any()
    keep, over = st.clone(), st.clone()
    clean = {k: t if t is None or t.dim() < 3 else torch.nan_to_num(t) for k, t in x.items()}
    out = dconv.dconv_scan(**x, state=over, lengths=ln, state_out=over)                   # over the state that it reads
    _check_scan(clean, keep, lengths, True, dt, out, over)
    got = dconv.dconv_scan_grad(dout, **x, state=keep, lengths=ln, dstate_out=dlast)
    _check_grads(clean, keep, torch.nan_to_num(dout), dlast, lengths, True, dt, got)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,C,S,G", [(1, 1, 1, 1), (1, 64, 16, 1), (5, 67, 5, 1), (3, 300, 32, 3), (300, 24, 8, 2), (7, 33, 4, 3)])
def test_steps(N, C, S, G, dtype):
    dt, M, T = TYPES[dtype], N + 3, 3
    x, _, _, _ = _inputs(N + C, dt, N, T, C, S, G)
    cache = torch.randn((M, C, S), generator=torch.Generator().manual_seed(5)).cuda()
    slots = torch.randperm(M, generator=torch.Generator().manual_seed(6))[:N].to(torch.int32)
    if N > 4:
        slots[1], slots[2], slots[3], slots[4] = -1, M, slots[0], 2147483647
    live = [n for n in range(N) if 0 <= slots[n] < M and slots[n] not in slots[:n]]
    before = cache.clone()
    start = torch.zeros((N, C, S), device="cuda")
    for n in live:
        start[n] = cache[slots[n]]
    outs = []
    for t in range(T):
        out = torch.full((N, C), NAN, dtype=dt, device="cuda")
        one = {k: v if v is None or k in ("A", "D", "delta_bias") else v[:, t] for k, v in x.items()}
        dconv.dconv_scan_step(**one, state=cache, slots=slots.cuda(), out=out)
        outs.append(out)
    outs = torch.stack(outs, 1)
    after = start.clone()
    for n in live:
        after[n] = cache[slots[n]]
        before[slots[n]] = cache[slots[n]]
    assert torch.equal(cache, before)                    # no other state changed
    _check_scan(x, start, [T if n in live else 0 for n in range(N)], True, dt, outs, after)


def test_extreme_steps_and_gates():
    """Steps that underflow and that decay everything, gates far out, a decay of exactly 1."""
    N, L, C, S = 1, 20, 64, 16
    x, st, dout, dlast = _inputs(9, torch.float32, N, L, C, S, 1, bias=False)
    x["delta"][0, :, 0] = -80.0
    x["delta"][0, :, 1] = 60.0
    x["delta"][0, :, 2] = 20.0001
    x["delta"][0, :, 3] = -17.5                          # 1 + e^x is 1 + 2^-25
    x["z"][0, :, 4] = 100.0
    x["z"][0, :, 5] = -100.0
    x["A"][6] = 0.0
    out = dconv.dconv_scan(**x, state=st)
    # the sigmoid of -100, 4e-44, is below the normal numbers of fp32 and 0 there (e^100 is infinite): 4e-44 times a gate of 100
    # and sums of up to 1e4
    _check_scan(x, st, None, True, torch.float32, out, None, 1e-30)
    _check_grads(x, st, dout, dlast, None, True, torch.float32, dconv.dconv_scan_grad(dout, **x, state=st, dstate_out=dlast), 1e-30)


def test_rows_beyond_32_bits():
    N, L, C, S = 2, 18, 64, 16
    big = torch.empty(((1 << 31) + (1 << 16),), dtype=torch.float16, device="cuda")
    at = lambda k: torch.as_strided(big, (N, L, C), ((1 << 31) - 100, 640, 1), 64 * k)
    x, st, dout, _ = _inputs(1, torch.float16, N, L, C, S, 1)
    far = dict(x)
    for k, name in enumerate(("u", "delta", "z")):
        far[name] = at(k).copy_(x[name])
    assert torch.equal(dconv.dconv_scan(**far, out=at(4)), dconv.dconv_scan(**x))
    a = dconv.dconv_scan_grad(at(5).copy_(dout), **far, du=at(6), ddelta=at(7), dz=at(8))
    b = dconv.dconv_scan_grad(dout, **x)
    for name in NAMES:
        if getattr(b, name) is not None:
            assert torch.equal(getattr(a, name), getattr(b, name)), name


def test_states_alone():
    """The C entry without an output: the state that a prompt leaves, and the starts."""
    from paper_1705_10591_amd import sequence as q
    N, L, C, S = 2, 50, 40, 16
    x, st, dout, _ = _inputs(2, torch.bfloat16, N, L, C, S, 1)
    last, starts = torch.empty((N, C, S), device="cuda"), dconv.scan_starts(N, L, C, S)
    dconv.dconv_scan(**x, state=st, state_out=last, starts=starts)
    only, begin = torch.full_like(last, NAN), torch.full_like(starts, NAN)
    rows = lambda t: (t.data_ptr(), *t.stride()[:2], 0)
    head = (1, N, L, C, S, 1, 0, 1, *rows(x["u"]), *rows(x["delta"]), *q._NONE, *q._NONE, *rows(x["B"]), *(7 * q._NONE),
            x["A"].data_ptr(), 0, x["delta_bias"].data_ptr(), st.data_ptr(), only.data_ptr(), 0, 0, 0, 0, 0, begin.data_ptr(), 0, 0)
    lib = dconv.load_library()
    need = lib.dconv_scan_workspace(q._SCAN.pack(*head, 0, 0), 0)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert lib.dconv_scan(q._SCAN.pack(*head, ws.data_ptr(), need), torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert torch.equal(only, last) and torch.equal(begin, starts)


def test_captured_calls_replay():
    N, L, C, S = 1, 300, 72, 16                          # with chunks
    x, st, dout, dlast = _inputs(4, torch.bfloat16, N, L, C, S, 1)
    cache = st.clone()

    def calls(out, last):
        dconv.dconv_scan(**x, state=st, out=out, state_out=last)
        one = {k: v if v is None or k in ("A", "D", "delta_bias") else v[:, 0] for k, v in x.items()}
        dconv.dconv_scan_step(**one, state=cache)
        return dconv.dconv_scan_grad(dout, **x, state=st, dstate_out=dlast)

    out, last = torch.empty((N, L, C), device="cuda", dtype=torch.bfloat16), torch.empty_like(st)
    eager = calls(out, last)
    want, wlast, moved = out.clone(), last.clone(), cache.clone()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
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
        assert torch.equal(dconv.dconv_scan(**x, state=st), want)


def test_calls_on_another_stream():
    x, st, dout, dlast = _inputs(6, torch.float32, 1, 300, 72, 8, 1)
    want, grads = dconv.dconv_scan(**x, state=st), dconv.dconv_scan_grad(dout, **x, state=st)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        a = dconv.dconv_scan(**x, state=st)
        b = dconv.dconv_scan_grad(dout, **x, state=st)
    c = dconv.dconv_scan(**x, state=st)                  # at the same time, with a workspace of its own
    torch.cuda.synchronize()
    assert torch.equal(a, want) and torch.equal(c, want) and all(torch.equal(p, q) for p, q in zip(b, grads))


@pytest.mark.parametrize("dtype", TYPES)
def test_a_layer_on_prompts_pieces_and_tokens(dtype):
    """Convolution and scan as a layer runs them: a prompt whole, in two pieces that hand their states on, and its end one
    token at a time from a cache; padded batch.  Pieces begin with rounded rows and fp32 states, as the whole has them there, so
    they agree to a step of the type, and of the scan's roundings."""
    dt = TYPES[dtype]
    N, L, C, S, F = 3, 90, 72, 16, 4
    g = torch.Generator().manual_seed(11)
    x, st, _, _ = _inputs(12, dt, N, L, C, S, 1, state=False)
    w, b = (0.5 * torch.randn((C, F), generator=g)).to(dt).cuda(), torch.randn(C, generator=g).to(dt).cuda()
    v = {k: x[k] for k in ("A", "D", "delta_bias")}
    tokens = lambda lo, hi: {k: x[k][:, lo:hi] for k in ("delta", "B", "C", "z")}
    lengths = torch.tensor([90, 64, 71], dtype=torch.int32, device="cuda")

    def layer(lo, hi, rows, h):
        ln = torch.clamp(lengths - lo, 0, hi - lo).to(torch.int32)
        c = dconv.dconv_causal(x["u"][:, lo:hi], w, b, state=rows, lengths=ln, state_out=rows)
        return dconv.dconv_scan(u=c, **tokens(lo, hi), **v, state=h, lengths=ln, state_out=h), c

    zero = lambda: (torch.zeros((N, F - 1, C), dtype=dt, device="cuda"), torch.zeros((N, C, S), device="cuda"))
    rows, h = zero()
    whole, conv = layer(0, L, rows, h)
    want = dict(x, u=conv)
    _check_scan(want, None, lengths.tolist(), True, dt, whole, h)
    rows2, h2 = zero()
    parts = [layer(lo, hi, rows2, h2) for lo, hi in ((0, 33), (33, 60))]
    out = torch.cat([p[0] for p in parts], 1)
    cache_rows, cache_h = torch.zeros((5, F - 1, C), dtype=dt, device="cuda"), torch.zeros((5, C, S), device="cuda")
    slots = torch.tensor([4, 0, 2], device="cuda")
    cache_rows[slots], cache_h[slots] = rows2, h2
    steps = []
    for t in range(60, L):
        live = torch.where(t < lengths, slots, -1).to(torch.int32)
        c = dconv.dconv_causal_step(x["u"][:, t], cache_rows, w, b, slots=live)
        steps.append(dconv.dconv_scan_step(u=c, **{k: q[:, 0] for k, q in tokens(t, t + 1).items()}, **v, state=cache_h, slots=live))
    out = torch.cat([out, torch.stack(steps, 1)], 1)
    _check_scan(want, None, lengths.tolist(), True, dt, out, cache_h[slots])
    assert torch.equal(cache_rows[slots], rows)


def test_a_layer_trains():
    """Gradients through both operators in a row against differences of the whole, in single precision."""
    N, L, C, S, F = 2, 37, 20, 8, 4
    x, _, dout, _ = _inputs(13, torch.float32, N, L, C, S, 1, state=False)
    g = torch.Generator().manual_seed(14)
    w, b = (0.5 * torch.randn((C, F), generator=g)).cuda(), torch.randn(C, generator=g).cuda()
    rest = {k: t for k, t in x.items() if k != "u"}
    c = dconv.dconv_causal(x["u"], w, b)
    sg = dconv.dconv_scan_grad(dout, u=c, **rest)
    cg = dconv.dconv_causal_grad(sg.du, x["u"], w, b)

    def value(xv, wv, av):
        conv = ref.causal(xv, wv, _np(b))[0]
        v = _reference(dict(x, u=x["u"]))
        v.update(u=conv, A=av)
        return (ref.scan(**v)[0] * _np(dout)).sum()

    base = [_np(x["u"]), _np(w), _np(x["A"])]
    rng = np.random.default_rng(0)
    for k, got in enumerate((cg.dx, cg.dfilt, sg.dA)):
        way = rng.standard_normal(base[k].shape)
        e = 1e-6
        plus, minus = list(base), list(base)
        plus[k], minus[k] = base[k] + e * way, base[k] - e * way
        diff = (value(*plus) - value(*minus)) / (2 * e)
        # differences in 64 bits are good to 1e-7 here; the gradients' own errors are below 1e-5 of the sizes that they add up
        assert abs(diff - (_np(got) * way).sum()) < 1e-5 * (np.abs(_np(got) * way)).sum() + 1e-6, k


def test_replays_read_lengths_and_slots_anew():
    """A captured step and prompt serve other rows and lengths on every replay."""
    N, L, C, S, F, M = 4, 40, 68, 16, 4, 9
    x, _, dout, _ = _inputs(21, torch.bfloat16, N, L, C, S, 1, state=False)
    g = torch.Generator().manual_seed(3)
    w = (0.5 * torch.randn((C, F), generator=g)).bfloat16().cuda()
    win0, h0 = torch.randn((M, F - 1, C), generator=g).bfloat16().cuda(), torch.randn((M, C, S), generator=g).cuda()
    one = {k: v if v is None or k in ("A", "D", "delta_bias") else v[:, 0] for k, v in x.items()}
    lengths, slots = torch.zeros(N, dtype=torch.int32, device="cuda"), torch.zeros(N, dtype=torch.int32, device="cuda")

    def calls(win, h):
        c = dconv.dconv_causal(x["u"], w, lengths=lengths)
        y = dconv.dconv_scan(**dict(x, u=c), lengths=lengths)
        grads = dconv.dconv_scan_grad(dout, **dict(x, u=c), lengths=lengths)
        u1 = dconv.dconv_causal_step(one["u"], win, w, slots=slots)
        y1 = dconv.dconv_scan_step(**dict(one, u=u1), state=h, slots=slots)
        return [c, y, u1, y1, win, h] + [t for t in grads if t is not None]

    win, h = win0.clone(), h0.clone()
    calls(win, h)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        captured = calls(win, h)
    for ln, sl in (([40, 1, 0, 17], [3, 1, 8, 0]), ([16, 33, 40, 5], [8, -1, 8, 2]), ([0, 0, 0, 0], [-1, 99, -5, 4])):
        lengths.copy_(torch.tensor(ln, dtype=torch.int32)), slots.copy_(torch.tensor(sl, dtype=torch.int32))
        win.copy_(win0), h.copy_(h0)
        graph.replay()
        torch.cuda.synchronize()
        eager = calls(win0.clone(), h0.clone())
        torch.cuda.synchronize()
        for k, (a, b) in enumerate(zip(captured, eager)):
            assert torch.equal(a, b), (ln, sl, k)


def test_inputs_that_share_memory():
    """Inputs repeated over sequences, tokens or groups by strides of zero."""
    N, L, C, S, G = 3, 21, 66, 8, 2
    x, st, dout, _ = _inputs(22, torch.float32, N, L, C, S, G)
    x["delta"] = x["delta"][:, :1].expand(N, L, C)
    x["z"] = x["z"][:1].expand(N, L, C)
    x["B"] = x["B"][:, :, :1].expand(N, L, G, S)
    x["C"] = x["C"][:1, :1].expand(N, L, G, S)
    dout = dout[:1].expand(N, L, C)
    full = {k: t if t is None else t.contiguous() for k, t in x.items()}
    assert torch.equal(dconv.dconv_scan(**x, state=st), dconv.dconv_scan(**full, state=st))
    for a, b in zip(dconv.dconv_scan_grad(dout, **x, state=st), dconv.dconv_scan_grad(dout.contiguous(), **full, state=st)):
        assert torch.equal(a, b)


def test_two_threads_on_streams_of_their_own():
    import threading
    x, st, dout, _ = _inputs(23, torch.bfloat16, 1, 300, 72, 16, 1)
    want, grads = dconv.dconv_scan(**x, state=st), dconv.dconv_scan_grad(dout, **x, state=st)
    torch.cuda.synchronize()
    wrong = []

    def work():
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(20):
                a, b = dconv.dconv_scan(**x, state=st), dconv.dconv_scan_grad(dout, **x, state=st)
            s.synchronize()
            if not (torch.equal(a, want) and all(torch.equal(p, q) for p, q in zip(b, grads))):
                wrong.append(1)

    threads = [threading.Thread(target=work) for _ in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
