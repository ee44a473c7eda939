"""Performance cases of the sequence operators: the short causal convolution over tokens and the selective scan
behind it, for prompts, in training and for one token at a time.

A case is a dict: `op`, the element type, N sequences of L tokens (or N rows of one token), C channels, F taps or S
states a channel, G groups of B and C, and what the call brings: a state from earlier tokens, sequences of different
lengths in a padded batch (`ragged`), a gate, slots of a cache of M rows.  Token tensors are slices of wider
projections, as in a model: x and the gate are halves of one product, B and C columns of another.
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _case(name, op, dtype, N, L, C, *, F=0, S=0, G=1, M=0, state=False, ragged=False, gate=False):
    return {"name": name, "op": op, "dtype": dtype, "N": N, "L": L, "C": C, "F": F, "S": S, "G": G, "M": M,
            "state": state, "ragged": ragged, "gate": gate}


def listed():
    return [
        # one token of one conversation: a call of a few microseconds, where latency is the time
        _case("causal_step_one", "causal_step", "bf16", 1, 1, 2048, F=4),
        # one token of each of 200 conversations whose windows lie anywhere in a cache of 256
        _case("causal_step_200_slots", "causal_step", "f16", 200, 1, 5120, F=4, M=256),
        # the next piece of seven prompts of different lengths, nothing a round number, three taps, single precision
        _case("causal_prompt_ragged", "causal", "f32", 7, 501, 1003, F=3, state=True, ragged=True),
        # a batch in training, bound by its half gigabyte of input and output
        _case("causal_prompt_large", "causal", "bf16", 8, 4096, 4096, F=4),
        # gradients of a small padded batch in single precision
        _case("causal_grad_ragged", "causal_grad", "f32", 3, 1021, 771, F=4, state=True, ragged=True),
        # gradients of a training batch
        _case("causal_grad_large", "causal_grad", "bf16", 8, 2048, 4096, F=4),
        # one token of one conversation
        _case("scan_step_one", "scan_step", "bf16", 1, 1, 2048, S=16, gate=True),
        # one token of each of 200 conversations, 84 MB of states
        _case("scan_step_200_slots", "scan_step", "bf16", 200, 1, 5120, S=16, M=256, gate=True),
        # six prompts of different lengths with two groups of B and C, single precision, continued from a state
        _case("scan_prompt_ragged", "scan", "f32", 6, 701, 1500, S=8, G=2, state=True, ragged=True, gate=True),
        # one long prompt: few channels for the chip, many tokens
        _case("scan_prompt_long", "scan", "bf16", 1, 16384, 4096, S=16, gate=True),
        # gradients of a small padded batch, continued from a state
        _case("scan_grad_ragged", "scan_grad", "f16", 3, 333, 520, S=16, state=True, ragged=True, gate=True),
        # gradients of a training batch
        _case("scan_grad_large", "scan_grad", "bf16", 4, 2048, 4096, S=16, gate=True),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: prompts of one token to long ones, batches, gradients, steps of few or many rows."""
    while True:
        op = rng.choice(["causal", "causal_grad", "causal_step", "scan", "scan", "scan_grad", "scan_grad", "scan_step"])
        dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
        C = _log(rng, 64, 8192)
        if rng.random() < 0.7:
            C = max(64, C // 64 * 64)
        if op.endswith("step"):
            N, L = _log(rng, 1, 256), 1
        else:
            N = 1 if rng.random() < 0.3 else _log(rng, 1, 16)
            L = _log(rng, 1, 16384)
        c = _case("", op, dtype, N, L, C)
        if op.startswith("causal"):
            c["F"] = 4 if rng.random() < 0.6 else rng.choice([2, 3, 5, 6, 7, 8] if op == "causal_step" else [1, 2, 3, 5, 6, 7, 8])
        else:
            c["S"] = 16 if rng.random() < 0.6 else rng.choice([1, 2, 3, 4, 8, 12, 24, 32])
            c["gate"] = rng.random() < 0.8
            if rng.random() < 0.3:
                c["G"] = rng.choice([2, 3, 4])
                c["C"] = C = max(1, C // c["G"]) * c["G"]
        if L == 1:
            c["M"] = N + _log(rng, 1, 64) if op.endswith("step") and rng.random() < 0.5 else 0
        else:
            c["state"] = c["F"] != 1 and rng.random() < 0.4          # (one tap has no rows before the first)
            c["ragged"] = N > 1 and rng.random() < 0.5
        cost = N * L * C * max(1, c["S"]) * (2 if op == "scan_grad" else 1)
        # no dearer than the largest listed cases, in arithmetic and in memory
        if cost > 4 * 2048 * 4096 * 16 * (2 if op.startswith("scan") else 0.125) or work(c)["bytes"] > 5.4e8:
            continue
        del c["name"]
        return c


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def prepare(case, seed):
    """What a user's program has in hand.  Parameters as a model has them after its initialisation: filters of a
    uniform distribution of 1/sqrt(F), steps between 0.001 and 0.1, decays of 1 to S, a skip of about one."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _TYPES[case["dtype"]]
    N, L, C, F, S, G, M = (case[k] for k in ("N", "L", "C", "F", "S", "G", "M"))
    step, grad = case["op"].endswith("step"), case["op"].endswith("grad")
    st = {"case": case, "lengths": None, "state": None, "slots": None}
    rows = _randn(g, N, L, 2 * C).to(dt)                         # one product gives x (or u) and the gate
    x, z = rows[:, :, :C], rows[:, :, C:]
    if case["ragged"]:                                           # one row is full, one (of many) is padding alone
        n = torch.randint(1, L + 1, (N,), generator=g, device="cuda", dtype=torch.int32)
        n[0] = L
        if N > 4:
            n[-1] = 0
        st["lengths"] = n
    if grad:
        st["dout"] = _randn(g, N, L, C).to(dt)
    if M:
        st["slots"] = torch.randperm(M, generator=g, device="cuda")[:N].to(torch.int32)
    if case["op"].startswith("causal"):
        st["filt"] = ((torch.rand((C, F), generator=g, device="cuda") * 2 - 1) / math.sqrt(F)).to(dt)
        st["bias"] = ((torch.rand((C,), generator=g, device="cuda") * 2 - 1) / math.sqrt(F)).to(dt)
        st["x"] = x
        if step or case["state"]:
            st["state"] = _randn(g, M or N, F - 1, C).to(dt)
        if grad and case["state"]:
            st["dstate_out"] = _randn(g, N, F - 1, C).to(dt)
    else:
        st["u"], st["z"] = x, z if case["gate"] else None
        st["delta"] = (0.5 * _randn(g, N, L, C)).to(dt)
        bc = _randn(g, N, L, 2 * G * S).to(dt)                   # one product gives B and C
        st["B"] = bc[:, :, :G * S].unflatten(2, (G, S))
        st["C"] = bc[:, :, G * S:].unflatten(2, (G, S))
        st["A"] = -torch.arange(1, S + 1, device="cuda") * torch.exp(0.1 * _randn(g, C, S))
        st["D"] = 1 + 0.1 * _randn(g, C)
        first = torch.exp(torch.rand((C,), generator=g, device="cuda") * math.log(100.0) + math.log(0.001))
        st["delta_bias"] = first + torch.log(-torch.expm1(-first))
        if step or case["state"]:
            st["state"] = _randn(g, M or N, C, S)
        if grad and case["state"]:
            st["dstate_out"] = _randn(g, N, C, S)
    if step:
        for k in ("x", "u", "delta", "z", "B", "C"):
            if st.get(k) is not None:
                st[k] = st[k][:, 0]
    return st


def run(state):
    return _own(state) if own else _plain(state)


def _own(st):
    import paper_1705_10591_amd as dconv
    case, op, state = st["case"], st["case"]["op"], st["state"]
    if op == "causal_step":
        return dconv.dconv_causal_step(st["x"], state, st["filt"], st["bias"], slots=st["slots"]), state
    if op == "causal":
        last = None if state is None else torch.empty_like(state)
        y = dconv.dconv_causal(st["x"], st["filt"], st["bias"], state=state, lengths=st["lengths"], state_out=last)
        return y, last
    if op == "causal_grad":
        return tuple(dconv.dconv_causal_grad(st["dout"], st["x"], st["filt"], st["bias"], state=state,
                                             lengths=st["lengths"], dstate_out=st.get("dstate_out")))
    args = (st["u"], st["delta"], st["A"], st["B"], st["C"])
    opts = {"D": st["D"], "z": st["z"], "delta_bias": st["delta_bias"]}
    if op == "scan_step":
        return dconv.dconv_scan_step(*args, state, slots=st["slots"], **opts), state
    if op == "scan":
        last = None if state is None else torch.empty_like(state)
        y = dconv.dconv_scan(*args, state=state, lengths=st["lengths"], state_out=last, **opts)
        return y, last
    return tuple(dconv.dconv_scan_grad(st["dout"], *args, state=state, lengths=st["lengths"],
                                       dstate_out=st.get("dstate_out"), **opts))


# ---- plain forms: elementary operations in 32 bits, rounded once at the end ----------------------------------------

def _plain(st):
    return {"causal": _plain_causal, "causal_grad": _plain_causal_grad, "causal_step": _plain_causal_step,
            "scan": _plain_scan, "scan_grad": _plain_scan_grad, "scan_step": _plain_scan_step}[st["case"]["op"]](st)


def _keep(st):
    """[N, L, 1]: tokens that belong to their sequence."""
    N, L = st["case"]["N"], st["case"]["L"]
    if st["lengths"] is None:
        return None
    return (torch.arange(L, device="cuda")[None, :] < st["lengths"][:, None])[:, :, None]


def _masked(t, keep):
    return t if keep is None else torch.where(keep, t, torch.zeros((), dtype=t.dtype, device="cuda"))


def _window(st):
    """[N, F - 1 + L, C] in 32 bits: the rows before the first token and the tokens."""
    x, F = st["x"].float(), st["case"]["F"]
    before = x.new_zeros((x.shape[0], F - 1, x.shape[2])) if st["state"] is None else st["state"].float()
    return torch.cat([before, _masked(x, _keep(st))], 1)


def _taps(rows, filt, bias, F, L):
    s = bias.float().expand(rows.shape[0], L, -1).clone()
    for j in range(F):
        s.addcmul_(rows[:, j:j + L], filt[:, j].float())
    return s


def _last_rows(st):
    """Where the last F - 1 rows before the end of each sequence lie in its window."""
    case = st["case"]
    n = torch.full((case["N"],), case["L"], device="cuda") if st["lengths"] is None else st["lengths"].long()
    return n[:, None] + torch.arange(case["F"] - 1, device="cuda")[None, :]


def _plain_causal(st):
    F, L = st["case"]["F"], st["case"]["L"]
    rows = _window(st)
    s = _taps(rows, st["filt"], st["bias"], F, L)
    y = _masked(s * torch.sigmoid(s), _keep(st)).to(st["x"].dtype)
    if st["state"] is None:
        return y, None
    at = _last_rows(st)[:, :, None].expand(-1, -1, rows.shape[2])
    return y, rows.gather(1, at).to(st["x"].dtype)


def _plain_causal_grad(st):
    F, L = st["case"]["F"], st["case"]["L"]
    rows, filt = _window(st), st["filt"].float()
    s = _taps(rows, st["filt"], st["bias"], F, L)
    sig = torch.sigmoid(s)
    ds = _masked(st["dout"].float() * sig * (1 + s * (1 - sig)), _keep(st))
    drows = torch.zeros_like(rows)
    dfilt = torch.empty_like(filt)
    for j in range(F):
        drows[:, j:j + L].addcmul_(ds, filt[:, j])
        dfilt[:, j] = (ds * rows[:, j:j + L]).sum((0, 1), dtype=torch.float64)
    dbias = ds.sum((0, 1), dtype=torch.float64).float()
    if st["state"] is None:
        return drows[:, F - 1:].to(st["x"].dtype), dfilt, dbias, None
    at = _last_rows(st)[:, :, None].expand(-1, -1, rows.shape[2])
    drows.scatter_add_(1, at, st["dstate_out"].float())
    drows = drows.to(st["x"].dtype)
    dx = _masked(drows[:, F - 1:], _keep(st))
    return dx, dfilt, dbias, drows[:, :F - 1].contiguous()


def _plain_causal_step(st):
    state, x = st["state"], st["x"]
    at = torch.arange(x.shape[0], device="cuda") if st["slots"] is None else st["slots"].long()
    rows = torch.cat([state[at], x[:, None]], 1)
    s = (rows.float() * st["filt"].float().t()).sum(1) + st["bias"].float()
    state[at] = rows[:, 1:]
    return (s * torch.sigmoid(s)).to(x.dtype), state


def _steps(st):
    """delta after bias and softplus, 0 at tokens that do not count: there the state stays as it is."""
    d = st["delta"].float() + st["delta_bias"]
    return _masked(torch.where(d > 20, d, torch.log1p(torch.exp(torch.clamp(d, max=20.0)))), _keep(st))


def _heads(t, C):
    """[..., G, S] in 32 bits, given to the C / G channels of each group: [..., C, S]."""
    return t.float().repeat_interleave(C // t.shape[-2], -2)


def _states(st, d, u):
    """Decays and states after every token, [L, N, C, S]."""
    C = st["case"]["C"]
    a = torch.exp(d.transpose(0, 1)[..., None] * st["A"])
    h = (d * u).transpose(0, 1)[..., None] * _heads(st["B"].transpose(0, 1), C)
    if st["state"] is not None:
        h[0].addcmul_(a[0], st["state"])
    for t in range(1, h.shape[0]):
        h[t].addcmul_(a[t], h[t - 1])
    return a, h


def _plain_scan(st):
    C, keep = st["case"]["C"], _keep(st)
    u, d = _masked(st["u"].float(), keep), _steps(st)
    _, h = _states(st, d, u)
    last = None if st["state"] is None else h[-1].clone()
    y = h.mul_(_heads(_masked(st["C"], None if keep is None else keep[..., None]).transpose(0, 1), C)).sum(-1)
    y = y.transpose(0, 1) + st["D"] * u
    if st["z"] is not None:
        z = st["z"].float()
        y = y * z * torch.sigmoid(z)
    return _masked(y, keep).to(st["u"].dtype), last


def _plain_scan_grad(st):
    case, keep = st["case"], _keep(st)
    C, G, S, dt = case["C"], case["G"], case["S"], st["u"].dtype
    u, d = _masked(st["u"].float(), keep), _steps(st)
    dout = _masked(st["dout"].float(), keep)
    a, h = _states(st, d, u)
    Ct = _heads(st["C"].transpose(0, 1), C)
    dz, dy = None, dout
    if st["z"] is not None:
        z = st["z"].float()
        sig = torch.sigmoid(z)
        y = (h * Ct).sum(-1).transpose(0, 1) + st["D"] * u
        dz = _masked(dout * y * sig * (1 + z * (1 - sig)), keep).to(dt)
        dy = _masked(dout * z * sig, keep)
        del y
    dyt = dy.transpose(0, 1)[..., None]
    dC = (dyt * h).unflatten(2, (G, C // G)).sum(3).transpose(0, 1).to(dt).contiguous()
    g = Ct.mul_(dyt)
    if st["state"] is not None:
        g[-1] += st["dstate_out"]
    for t in range(g.shape[0] - 2, -1, -1):
        g[t].addcmul_(a[t + 1], g[t + 1])
    dstate = None if st["state"] is None else a[0] * g[0]
    # a := gradient of the decay's exponent, g a h_before
    a.mul_(g)
    a[1:].mul_(h[:-1])
    a[0].mul_(st["state"] if st["state"] is not None else 0.0)
    del h
    dA = (a * d.transpose(0, 1)[..., None]).sum((0, 1), dtype=torch.float64).float()
    dd = a.mul_(st["A"]).sum(-1).transpose(0, 1)
    dB = (g * (d * u).transpose(0, 1)[..., None]).unflatten(2, (G, C // G)).sum(3).transpose(0, 1)
    gB = g.mul_(_heads(st["B"].transpose(0, 1), C)).sum(-1).transpose(0, 1)
    du = _masked(d * gB + st["D"] * dy, keep).to(dt).contiguous()
    dd = _masked((dd + u * gB) * torch.sigmoid(st["delta"].float() + st["delta_bias"]), keep)
    dD = (dy * u).sum((0, 1), dtype=torch.float64).float()
    dbias = dd.sum((0, 1), dtype=torch.float64).float()
    return du, dd.to(dt).contiguous(), dA, dB.to(dt).contiguous(), dC, dD, dz, dbias, dstate


def _plain_scan_step(st):
    state, u = st["state"], st["u"].float()
    C = st["case"]["C"]
    at = torch.arange(u.shape[0], device="cuda") if st["slots"] is None else st["slots"].long()
    d = st["delta"].float() + st["delta_bias"]
    d = torch.where(d > 20, d, torch.log1p(torch.exp(torch.clamp(d, max=20.0))))[..., None]
    h = torch.exp(d * st["A"]) * state[at] + d * u[..., None] * _heads(st["B"], C)
    state[at] = h
    y = (h * _heads(st["C"], C)).sum(-1) + st["D"] * u
    if st["z"] is not None:
        z = st["z"].float()
        y = y * z * torch.sigmoid(z)
    return y.to(st["u"].dtype), state


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    if case["op"].startswith("causal"):
        return _exact_causal(st)
    return _exact_scan(st)


def _lengths(st):
    case = st["case"]
    return [case["L"]] * case["N"] if st["lengths"] is None else st["lengths"].tolist()


def _exact_causal(st):
    """Every sequence by itself: its rows, the taps one by one; gradients by differentiation of that."""
    case, op = st["case"], st["case"]["op"]
    F, C = case["F"], case["C"]
    filt, bias = st["filt"].double(), st["bias"].double()
    x = st["x"].double()
    if op == "causal_step":
        x = x[:, None]
        slots = range(case["N"]) if st["slots"] is None else st["slots"].tolist()
        before, state = st["state"].double()[list(slots)], st["state"].double().clone()
    else:
        slots = range(case["N"])
        before = x.new_zeros((case["N"], F - 1, C)) if st["state"] is None else st["state"].double()
        state = before.clone()
    grad = op == "causal_grad"
    y, dx, dstate = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(before)
    if grad:
        filt.requires_grad_(), bias.requires_grad_()
        dout = st["dout"].double()
        dfilt, dbias = torch.zeros_like(filt), torch.zeros_like(bias)
    for n, (len_, slot) in enumerate(zip(_lengths(st), slots)):
        rows = torch.cat([before[n], x[n, :len_]]).requires_grad_(grad)
        s = bias.expand(len_, C)
        for j in range(F):
            s = s + filt[:, j] * rows[j:j + len_]
        out = s / (1 + torch.exp(-s))
        if not grad:
            y[n, :len_] = out
            state[slot] = rows[len_:]
            continue
        total = (out * dout[n, :len_]).sum()
        if st["state"] is not None:
            total = total + (rows[len_:] * st["dstate_out"][n].double()).sum()
        dr, df, db = torch.autograd.grad(total, (rows, filt, bias), allow_unused=True)
        dstate[n], dx[n, :len_] = dr[:F - 1], dr[F - 1:]
        dfilt += 0 if df is None else df
        dbias += 0 if db is None else db
    none = st["state"] is None
    if grad:
        return dx, dfilt, dbias, None if none else dstate
    if op == "causal_step":
        return y[:, 0], state
    return y, None if none else state


def _prefix(a, b):
    """h[t] = a[t] h[t-1] + b[t] along the first axis, by doubling: after each round every element holds what twice as
    many tokens before it bring."""
    k = 1
    while k < b.shape[0]:
        b = torch.cat([b[:k], b[k:] + a[k:] * b[:-k]])
        a = torch.cat([a[:k], a[k:] * a[:-k]])
        k *= 2
    return b


def _exact_scan(st):
    """A few channels of a sequence at a time; gradients by differentiation."""
    case, op = st["case"], st["case"]["op"]
    N, C, S, G = case["N"], case["C"], case["S"], case["G"]
    step, grad = op == "scan_step", op == "scan_grad"
    wide = {k: st[k].double()[:, None] if step else st[k].double() for k in ("u", "delta", "B", "C")}
    gate = None if st["z"] is None else (st["z"].double()[:, None] if step else st["z"].double())
    A, skip, bias = (st[k].double() for k in ("A", "D", "delta_bias"))
    slots = st["slots"].tolist() if st["slots"] is not None else list(range(N))
    state = torch.zeros((N, C, S), dtype=torch.float64, device="cuda") if st["state"] is None else st["state"].double()
    last = state.clone()
    y = torch.zeros_like(wide["u"])
    if grad:
        dout = st["dout"].double()
        d = {k: torch.zeros_like(v) for k, v in wide.items()}
        d["z"] = None if gate is None else torch.zeros_like(gate)
        d.update(A=torch.zeros_like(A), D=torch.zeros_like(skip), bias=torch.zeros_like(bias), state=torch.zeros_like(state))
    for n, len_ in enumerate(_lengths(st)):
        if len_ == 0:
            if grad and st["state"] is not None:
                d["state"][n] = st["dstate_out"][n].double()
            continue
        width = max(1, (1 << 24 if grad else 1 << 27) // (len_ * S))
        for grp in range(G):
            for lo in range(grp * (C // G), (grp + 1) * (C // G), width):
                ch = slice(lo, min(lo + width, (grp + 1) * (C // G)))
                v = [wide["u"][n, :len_, ch], wide["delta"][n, :len_, ch], wide["B"][n, :len_, grp],
                     wide["C"][n, :len_, grp], A[ch], skip[ch], bias[ch], state[slots[n], ch]]
                if gate is not None:
                    v.append(gate[n, :len_, ch])
                if grad:
                    v = [t.detach().clone().requires_grad_() for t in v]
                u, delta, Bt, Ct, a_, skip_, bias_, h0 = v[:8]
                raw = delta + bias_
                dt = torch.clamp(raw, min=0) + torch.log1p(torch.exp(-torch.abs(raw)))
                decay = torch.exp(dt[..., None] * a_)
                b = (dt * u)[..., None] * Bt[:, None, :]
                b = torch.cat([(b[0] + decay[0] * h0)[None], b[1:]])
                h = _prefix(decay, b)
                out = (h * Ct[:, None, :]).sum(-1) + skip_ * u
                if gate is not None:
                    out = out * v[8] / (1 + torch.exp(-v[8]))
                if not grad:
                    y[n, :len_, ch] = out
                    last[slots[n], ch] = h[-1]
                    continue
                total = (out * dout[n, :len_, ch]).sum()
                if st["state"] is not None:
                    total = total + (h[-1] * st["dstate_out"][n, ch].double()).sum()
                r = torch.autograd.grad(total, v)
                d["u"][n, :len_, ch], d["delta"][n, :len_, ch] = r[0], r[1]
                d["B"][n, :len_, grp] += r[2]
                d["C"][n, :len_, grp] += r[3]
                d["A"][ch] += r[4]
                d["D"][ch] += r[5]
                d["bias"][ch] += r[6]
                d["state"][n, ch] = r[7]
                if gate is not None:
                    d["z"][n, :len_, ch] = r[8]
    none = st["state"] is None
    if grad:
        return (d["u"], d["delta"], d["A"], d["B"], d["C"], d["D"], d["z"], d["bias"], None if none else d["state"])
    if step:
        return y[:, 0], last
    return y, None if none else last


def work(case):
    """Each input read once, each output written once; a multiply and an add per tap, and per state of the scan the
    decay's product, its exponential, the input's product and two multiply-adds (three times that for gradients)."""
    N, L, C, F, S, G = (case[k] for k in ("N", "L", "C", "F", "S", "G"))
    e = 4 if case["dtype"] == "f32" else 2
    rows, op, st = N * L * C, case["op"], int(case["state"])
    if op == "causal":
        return {"bytes": e * (2 * rows + C * (F + 1) + 2 * st * N * (F - 1) * C), "flops": 2 * F * rows + 4 * rows}
    if op == "causal_grad":
        return {"bytes": e * (3 * rows + C * (F + 1) + 3 * st * N * (F - 1) * C) + 4 * C * (F + 1),
                "flops": 6 * F * rows + 8 * rows}
    if op == "causal_step":
        return {"bytes": e * (2 * rows + C * (F + 1) + 2 * N * (F - 1) * C), "flops": 2 * F * rows + 4 * rows}
    gate, bc, per = int(case["gate"]), N * L * G * S, N * C * S
    if op == "scan_grad":
        return {"bytes": e * ((5 + 2 * gate) * rows + 4 * bc) + 8 * C * (S + 2) + 4 * 3 * st * per,
                "flops": 21 * rows * S + 20 * rows}
    kept = 2 if op == "scan_step" else 2 * st
    return {"bytes": e * ((3 + gate) * rows + 2 * bc) + 4 * C * (S + 2) + 4 * kept * per, "flops": 7 * rows * S + 10 * rows}
