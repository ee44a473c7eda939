"""The kernels of the operators over tokens that sizes choose: strips of every length, scans of one pass and of chunks."""
import pytest
import torch

import paper_1705_10591_amd as dconv
from test_causal_gpu import NAN, TYPES
from test_causal_gpu import _check_grads as _check_causal_grads
from test_causal_gpu import _inputs as _causal_inputs
from test_scan_gpu import NAMES, _check_grads, _check_scan, _inputs

pytestmark = pytest.mark.gpu


def _lengths(N, L):
    n = [L, L // 2, 0, 1, L - 1, 33 % L, L, (L * 2 // 3) | 1]
    return torch.tensor([n[k % len(n)] for k in range(N)], dtype=torch.int32, device="cuda")


# strips of 16 and 32 tokens (calls of fewer runs have strips of 8), with a last one that is cut; whole runs and cut ones
@pytest.mark.parametrize("dtype,N,L,C,F", [("bf16", 8, 1021, 4104, 4), ("bf16", 8, 2037, 4101, 8), ("f32", 8, 2037, 2053, 3),
                                           ("f16", 8, 1021, 4104, 1)])
def test_long_strips(dtype, N, L, C, F):
    """The bits of the same channels in calls of few, which have short strips."""
    x, w, b, st, _, _ = _causal_inputs(L + C, TYPES[dtype], N, L, C, F)
    ln, last = _lengths(N, L), torch.empty_like(st)
    out = dconv.dconv_causal(x, w, b, state=st, lengths=ln, state_out=last)
    for lo in range(0, C, 512):
        s = slice(lo, lo + 512)
        one = torch.empty_like(st[:, :, s], memory_format=torch.contiguous_format)
        want = dconv.dconv_causal(x[:, :, s], w[s], b[s], state=st[:, :, s].contiguous(), lengths=ln, state_out=one)
        assert torch.equal(out[:, :, s], want) and torch.equal(last[:, :, s], one), lo


# strips of 16, 32, 64 and 128; workgroups of up to 32 runs and of 64
@pytest.mark.parametrize("dtype,N,L,C,F", [("bf16", 8, 250, 4096, 4), ("bf16", 8, 507, 4096, 8), ("bf16", 8, 1021, 4096, 4),
                                           ("bf16", 8, 2037, 4098, 4), ("f32", 8, 1021, 8193, 3), ("f16", 8, 2037, 8197, 4),
                                           ("f32", 8, 2037, 4096, 1)])
def test_long_strips_of_gradients(dtype, N, L, C, F):
    x, w, b, st, dout, dlast = _causal_inputs(L + C, TYPES[dtype], N, L, C, F)
    ln = _lengths(N, L)
    got = dconv.dconv_causal_grad(dout, x, w, b, state=st, lengths=ln, dstate_out=dlast)
    tokens = int(ln.sum())
    step = 510 + C % 2                                   # pieces of the call's parity: even and odd ones have kernels of their own
    for lo in range(0, C, step):
        s = slice(lo, lo + step)
        if (min(lo + step, C) - lo) % 2 != C % 2:
            s = slice(lo - 1, lo + step)
        piece = lambda t: t[:, :, s]
        want = dconv.dconv_causal_grad(piece(dout), piece(x), w[s], b[s], state=piece(st).contiguous(), lengths=ln,
                                       dstate_out=piece(dlast).contiguous())
        assert torch.equal(piece(got.dx), want.dx) and torch.equal(piece(got.dstate), want.dstate), lo
        # the same terms in another order: values of up to about 30 (five sigmas of x times dout times silu'), sums that grow
        # like the root of their number; far below, a wrong or missing row is one of its own
        for name in ("dfilt", "dbias"):
            off = (getattr(got, name)[s] - getattr(want, name)).abs().max().item()
            assert off < 2.0 ** -24 * 8 * tokens ** 0.5 * 30, (name, lo, off)


@pytest.mark.parametrize("dtype", TYPES)
def test_the_gradient_of_the_last_rows_without_a_state(dtype):
    x, w, b, _, dout, dlast = _causal_inputs(3, TYPES[dtype], 3, 21, 70, 4)
    ln = torch.tensor([21, 2, 0], dtype=torch.int32, device="cuda")
    _check_causal_grads(dout, x, w, b, None, ln, ln.tolist(), dlast, True, TYPES[dtype])


def _check_all(x, st, dout, dlast, lengths, dt):
    N, L, C = x["u"].shape
    S, G = x["A"].shape[1], x["B"].shape[2]
    ln = None if lengths is None else lengths.tolist()
    last, starts = torch.full((N, C, S), NAN, device="cuda"), dconv.scan_starts(N, L, C, S, G)
    plain = dconv.dconv_scan(**x, state=st, lengths=lengths, state_out=last)
    _check_scan(x, st, ln, True, dt, plain, last)
    out = dconv.dconv_scan(**x, state=st, lengths=lengths, state_out=last, starts=starts)
    assert torch.equal(out, plain)
    again = dconv.dconv_scan_grad(dout, **x, state=st, lengths=lengths, dstate_out=dlast)
    _check_grads(x, st, dout, dlast, ln, True, dt, again)
    kept = dconv.dconv_scan_grad(dout, **x, state=st, lengths=lengths, dstate_out=dlast, starts=starts)
    _check_grads(x, st, dout, dlast, ln, True, dt, kept)
    return kept, again


# seven to nine tiles of 16 tokens are one pass with an output (six have B and C by way of LDS, ten are cut into chunks), whole
# blocks of 64 channels and cut ones, of one, two and four states a wave and of eight waves
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,L,C,S,G", [(2, 130, 70, 16, 1), (1, 112, 64, 6, 1), (2, 130, 128, 3, 2), (2, 144, 70, 20, 1), (1, 100, 192, 9, 3)])
def test_scans_of_one_pass(N, L, C, S, G, dtype):
    x, st, dout, dlast = _inputs(L + C + S, TYPES[dtype], N, L, C, S, G)
    _check_all(x, st, dout, dlast, None, TYPES[dtype])


# groups of one channel have a block each: as many as give the chip its waves without chunks, in prompts and gradients
@pytest.mark.parametrize("C,S", [(512, 16), (512, 8), (512, 1), (512, 4), (256, 32)])
def test_long_scans_of_one_pass(C, S):
    x, st, dout, dlast = _inputs(C + S, torch.float32, 1, 170, C, S, C)
    kept, again = _check_all(x, st, dout, dlast, None, torch.float32)
    for name in NAMES:                                   # no chunks: states made again are the same
        assert torch.equal(getattr(kept, name), getattr(again, name)), name


# (a gradient of fewer than six tiles has no chunks either)
@pytest.mark.parametrize("C,S,G", [(70, 16, 1), (64, 3, 1), (128, 32, 2), (40, 8, 2)])
def test_states_made_again_are_those_kept(C, S, G):
    x, st, dout, dlast = _inputs(C + S, torch.bfloat16, 3, 80, C, S, G)
    ln = torch.tensor([80, 17, 0], dtype=torch.int32, device="cuda")
    starts = dconv.scan_starts(3, 80, C, S, G)
    dconv.dconv_scan(**x, state=st, lengths=ln, starts=starts)
    for a, b in zip(*(dconv.dconv_scan_grad(dout, **x, state=st, lengths=ln, dstate_out=dlast, starts=k) for k in (starts, None))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("lo", [0, 1472, 1000])
def test_a_training_batch_of_one_pass(lo):
    """384 whole blocks of channels, ragged, with starts.  Channels are on their own but for dB and dC: 64 of them are looked at, in
    all sequences."""
    N, L, C, S = 16, 200, 1536, 16
    x, st, dout, dlast = _inputs(1, torch.bfloat16, N, L, C, S, 1)
    ln, s = _lengths(N, L), slice(lo, lo + 64)
    starts, last = dconv.scan_starts(N, L, C, S), torch.full((N, C, S), NAN, device="cuda")
    out = dconv.dconv_scan(**x, state=st, lengths=ln, state_out=last, starts=starts)
    got = dconv.dconv_scan_grad(dout, **x, state=st, lengths=ln, dstate_out=dlast, starts=starts)
    part = {k: t if k in ("B", "C") else t[s] if k in ("A", "D", "delta_bias") else t[:, :, s] for k, t in x.items()}
    first, final = st[:, s].contiguous(), dlast[:, s].contiguous()
    _check_scan(part, first, ln.tolist(), True, torch.bfloat16, out[:, :, s], last[:, s])
    small = dconv.dconv_scan_grad(dout[:, :, s], **part, state=first, lengths=ln, dstate_out=final)
    seen = {k: getattr(got, k)[:, :, s] for k in ("du", "ddelta", "dz")}
    seen.update({k: getattr(got, k)[s] for k in ("dA", "dD", "ddelta_bias")}, dstate=got.dstate[:, s])
    _check_grads(part, first, dout[:, :, s], final, ln.tolist(), True, torch.bfloat16, small._replace(**seen))


# chunks of few states, of whole blocks and cut ones, ragged, with states made again and kept
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("L,C,S,G", [(400, 70, 1, 1), (330, 64, 3, 1), (400, 128, 4, 1), (400, 64, 7, 1), (300, 64, 16, 1), (300, 128, 24, 2)])
def test_chunks(L, C, S, G, dtype):
    x, st, dout, dlast = _inputs(L + C + S, TYPES[dtype], 4, L, C, S, G)
    ln = torch.tensor([L, 0, 33, L - 17], dtype=torch.int32, device="cuda")
    _check_all(x, st, dout, dlast, ln, TYPES[dtype])
    x, _, dout, dlast = _inputs(L + C + S + 1, TYPES[dtype], 2, L, C, S, G, state=False)
    _check_all(x, None, dout, dlast, None, TYPES[dtype])                                  # a last state's gradient without a first state


# 1024 waves by themselves: chunks of 144 tokens, in prompts and in gradients
@pytest.mark.parametrize("L,S,grad", [(1152, 16, False), (864, 3, False), (576, 16, True), (576, 4, True)])
def test_long_chunks(L, S, grad):
    C = 256
    x, st, dout, dlast = _inputs(L + S, torch.float32, 1, L, C, S, C)
    last = torch.empty_like(st)
    if grad:
        _check_grads(x, st, dout, dlast, None, True, torch.float32, dconv.dconv_scan_grad(dout, **x, state=st, dstate_out=dlast))
    else:
        _check_scan(x, st, None, True, torch.float32, dconv.dconv_scan(**x, state=st, state_out=last), last)


@pytest.mark.parametrize("C,S", [(64, 32), (128, 17), (64, 24)])
def test_whole_blocks_of_eight_waves(C, S):
    for L in (20, 90, 120):
        x, st, dout, dlast = _inputs(L + S, torch.bfloat16, 2, L, C, S, 1)
        _check_all(x, st, dout, dlast, torch.tensor([L, L // 2], dtype=torch.int32, device="cuda"), torch.bfloat16)
