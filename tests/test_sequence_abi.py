"""What the operators over tokens refuse: C entries on the CPU (every call here fails before a launch), the Python functions
on tensors they cannot take."""
import ctypes

import pytest
import torch

import paper_1705_10591_amd as dconv
from paper_1705_10591_amd import sequence as q

P = 0x1000            # a pointer that is never followed
CAUSAL = ["dtype", "N", "L", "C", "F", "M", "silu", "reserved"] + [f"{t}.{f}" for t in ("x", "out", "dout", "dx") for f in ("p", "sn", "sl", "sg")] + \
    ["filt", "bias", "state", "state_out", "dstate_out", "dstate", "dfilt", "dbias", "lengths", "slots", "workspace", "workspace_bytes"]
SCAN = ["dtype", "N", "L", "C", "S", "G", "M", "softplus"] + \
    [f"{t}.{f}" for t in ("u", "delta", "z", "out", "B", "Cm", "dout", "du", "ddelta", "dz", "dB", "dC") for f in ("p", "sn", "sl", "sg")] + \
    ["A", "D", "delta_bias", "state", "state_out", "dstate_out", "dstate", "dA", "dD", "ddelta_bias", "starts", "lengths", "slots",
     "workspace", "workspace_bytes"]
OK, NULL, SHAPE, UNSUPPORTED, SCRATCH = (dconv.STATUS_OK, dconv.STATUS_NULL_POINTER, dconv.STATUS_BAD_SHAPE,
                                         dconv.STATUS_UNSUPPORTED, dconv.STATUS_SCRATCH_EXCEEDED)


def _pack(names, layout, values):
    assert set(values) <= set(names)
    return layout.pack(*(values.get(n, 0) for n in names))


def causal(name, **change):
    v = {"dtype": 1, "N": 2, "L": 1 if name.endswith("step") else 9, "C": 70, "F": 4, "M": 2, "silu": 1, "x.p": P, "out.p": P + 16,
         "dout.p": P, "dx.p": P + 16, "filt": P, "state_out": P, "dfilt": P, "workspace": P, "workspace_bytes": 1 << 40}
    v.update({k.replace("_p", ".p") if k in ("x_p", "out_p", "dout_p", "dx_p") else k: t for k, t in change.items()})
    return getattr(dconv.load_library(), name)(_pack(CAUSAL, q._CAUSAL, v), None)


def scan(name, **change):
    v = {"dtype": 1, "N": 2, "L": 1 if name.endswith("step") else 200, "C": 70, "S": 16, "G": 1, "M": 2, "softplus": 1, "A": P, "state_out": P,
         "dA": P, "workspace": P, "workspace_bytes": 1 << 50}
    v.update({t + ".p": P for t in ("u", "delta", "out", "B", "Cm", "dout", "du", "ddelta", "dB", "dC")})
    v.update({k.replace("_p", ".p") if k.endswith("_p") else k: t for k, t in change.items()})
    return getattr(dconv.load_library(), name)(_pack(SCAN, q._SCAN, v), None)


def test_structs_are_laid_out_as_in_the_header(tmp_path):
    """The packed bytes against the C compiler's offsets."""
    import re
    import subprocess
    from pathlib import Path
    header = Path(__file__).resolve().parent.parent / "include" / "dconv.h"
    lines = [f'printf("%zu\\n", offsetof({t}, {n}));' for t, names in (("dconv_causal_args", CAUSAL), ("dconv_scan_args", SCAN)) for n in names]
    lines += [f'printf("%zu\\n", sizeof({t}));' for t in ("dconv_causal_args", "dconv_scan_args")]
    src = tmp_path / "o.c"
    src.write_text(f'#include <stdio.h>\n#include <stddef.h>\n#include "{header}"\nint main(void) {{ {" ".join(lines)} return 0; }}')
    subprocess.run(["gcc", str(src), "-o", str(tmp_path / "o")], check=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "o")], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for names in (CAUSAL, SCAN):
        want += [4 * i for i in range(8)] + [32 + 8 * i for i in range(len(names) - 8)]
    assert got == want + [q._CAUSAL.size, q._SCAN.size]


@pytest.mark.parametrize("name", ["dconv_causal", "dconv_causal_grad", "dconv_causal_step"])
def test_causal_refusals(name):
    assert getattr(dconv.load_library(), name)(None, None) == NULL
    step, grad = name.endswith("step"), name.endswith("grad")
    needed = ["x_p", "filt"] + (["dout_p", "dx_p", "workspace"] if grad else ["out_p"]) + (["state_out"] if step else [])
    for k in needed:
        assert causal(name, **{k: 0}) == NULL, k
    for k in ("N", "L", "C", "F"):
        for v in (0, -1):
            assert causal(name, **{k: v}) == SHAPE, k
    assert causal(name, F=9) == SHAPE
    assert causal(name, L=(1 << 30) + 1) == SHAPE
    assert causal(name, N=1, C=(1 << 30) + 1) == SHAPE
    assert causal(name, N=2147483647, C=2147483647, M=2147483647) == SHAPE           # more workgroups than a launch has
    for d in (2, 4, -1):
        assert causal(name, dtype=d) == UNSUPPORTED
    for k in needed + ["bias"]:
        if k != "workspace":
            assert causal(name, **{k: P + 1}) == SHAPE, k
    assert causal(name, dtype=3, x_p=P + 2) == SHAPE
    assert causal(name, lengths=P + 2) == SHAPE
    if not step:
        assert causal(name, **{"dx_p" if grad else "out_p": P}) == SHAPE       # over x
    if step:
        assert causal(name, L=2) == SHAPE
        assert causal(name, M=1) == SHAPE                    # fewer windows than rows, no slots
        assert causal(name, M=0, slots=P) == SHAPE
    if grad:
        need = dconv.load_library().dconv_causal_workspace(_pack(CAUSAL, q._CAUSAL, {"dtype": 1, "N": 2, "L": 9, "C": 70, "F": 4}))
        assert need > 0 and causal(name, workspace_bytes=need - 1) == SCRATCH
        assert causal(name, workspace=P + 8) == SHAPE


@pytest.mark.parametrize("name", ["dconv_scan", "dconv_scan_grad", "dconv_scan_step"])
def test_scan_refusals(name):
    assert getattr(dconv.load_library(), name)(None, None) == NULL
    step, grad = name.endswith("step"), name.endswith("grad")
    needed = ["u_p", "delta_p", "B_p", "A", "Cm_p"]
    needed += ["dout_p", "du_p", "ddelta_p", "dB_p", "dC_p", "dA"] if grad else ["state_out"] if step else []
    for k in needed + ([] if step else ["workspace"]) + (["out_p"] if step else []):
        assert scan(name, **{k: 0}) == NULL, k
    if name == "dconv_scan":
        assert scan(name, out_p=0, state_out=0, starts=0) == NULL              # nothing to be made
    if grad:
        assert scan(name, z_p=P) == NULL                                       # a gate without a place for its gradient
    for k in ("N", "L", "C", "S", "G"):
        for v in (0, -1):
            assert scan(name, **{k: v}) == SHAPE, k
    assert scan(name, S=33) == SHAPE
    assert scan(name, G=3) == SHAPE                                            # 70 channels in 3 groups
    assert scan(name, L=(1 << 30) + 1) == SHAPE
    assert scan(name, N=1, C=(1 << 30) + 1) == SHAPE
    assert scan(name, N=1 << 30, C=1 << 30, M=1 << 30) == SHAPE
    for d in (2, 4, -1):
        assert scan(name, dtype=d) == UNSUPPORTED
    for k in needed:
        assert scan(name, **{k: P + 1}) == SHAPE, k
    assert scan(name, dtype=3, u_p=P + 2) == SHAPE
    for k in ("D", "delta_bias", "state", "lengths", "slots"):
        assert scan(name, **{k: P + 2}) == SHAPE, k
    if step:
        assert scan(name, L=2) == SHAPE
        assert scan(name, M=1) == SHAPE
        assert scan(name, M=0, slots=P) == SHAPE
    else:
        lib = dconv.load_library()
        sizes = _pack(SCAN, q._SCAN, {"dtype": 1, "N": 2, "L": 200, "C": 70, "S": 16, "G": 1, "out.p": P})
        need = lib.dconv_scan_workspace(sizes, int(grad))
        assert need > 0 and scan(name, workspace_bytes=need - 1) == SCRATCH
        assert scan(name, workspace=P + 8) == SHAPE
        assert scan(name, starts=P + 8) == SHAPE


def test_sizes_of_workspaces():
    lib = dconv.load_library()
    bad = _pack(SCAN, q._SCAN, {"dtype": 1, "N": 2, "L": 0, "C": 70, "S": 16, "G": 1})
    assert lib.dconv_scan_workspace(bad, 0) == lib.dconv_scan_workspace(bad, 1) == lib.dconv_scan_starts(bad) == -1
    assert lib.dconv_causal_workspace(_pack(CAUSAL, q._CAUSAL, {"dtype": 1, "N": 1, "L": 1, "C": 1, "F": 9})) == -1
    assert lib.dconv_scan_starts(None) == lib.dconv_scan_workspace(None, 1) == lib.dconv_causal_workspace(None) == -1
    # a short prompt needs none for its output, but for the states alone
    short = {"dtype": 1, "N": 2, "L": 9, "C": 70, "S": 16, "G": 1}
    assert lib.dconv_scan_workspace(_pack(SCAN, q._SCAN, {**short, "out.p": P}), 0) == 0
    assert lib.dconv_scan_workspace(_pack(SCAN, q._SCAN, short), 0) > 0
    # sizes that pass 32 bits
    big = _pack(SCAN, q._SCAN, {"dtype": 1, "N": 64, "L": 1 << 17, "C": 8192, "S": 16, "G": 1})
    assert lib.dconv_scan_starts(big) == 64 * (1 << 13) * 8192 * 16 * 4
    assert lib.dconv_scan_workspace(big, 1) > lib.dconv_scan_starts(big)


def test_python_functions_refuse_cpu_tensors():
    x, w = torch.zeros(1, 4, 8), torch.zeros(8, 4)
    for call in (lambda: dconv.dconv_causal(x, w), lambda: dconv.dconv_causal_grad(x, x, w),
                 lambda: dconv.dconv_causal_step(x[0], torch.zeros(4, 3, 8), w),
                 lambda: dconv.dconv_scan(x, x, w, x, x), lambda: dconv.dconv_scan_grad(x, x, x, w, x, x),
                 lambda: dconv.dconv_scan_step(x[0], x[0], w, x, x, x)):
        with pytest.raises(TypeError):
            call()


@pytest.mark.gpu
def test_python_functions_refuse_what_does_not_fit():
    dev = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t, device="cuda")
    x, w, b = dev(2, 9, 8), dev(8, 4), dev(8)
    refused = [
        (TypeError, lambda: dconv.dconv_causal(x.double(), w)),
        (TypeError, lambda: dconv.dconv_causal(x[0], w)),
        (TypeError, lambda: dconv.dconv_causal(x, w.float())),
        (TypeError, lambda: dconv.dconv_causal(x.transpose(1, 2), dev(9, 4))),                 # channels apart
        (TypeError, lambda: dconv.dconv_causal(x, dev(8, 8)[:, ::2])),
        (ValueError, lambda: dconv.dconv_causal(x, dev(7, 4))),
        (ValueError, lambda: dconv.dconv_causal(x, w, dev(7))),
        (ValueError, lambda: dconv.dconv_causal(x, w, state=dev(2, 4, 8))),
        (ValueError, lambda: dconv.dconv_causal(x, w, out=dev(2, 9, 7))),
        (ValueError, lambda: dconv.dconv_causal(x, w, out=dev(1, 9, 8).expand(2, 9, 8))),      # sequences on top of each other
        (TypeError, lambda: dconv.dconv_causal(x, w, lengths=dev(2, t=torch.int64))),
        (ValueError, lambda: dconv.dconv_causal(x, w, lengths=dev(3, t=torch.int32))),
        (TypeError, lambda: dconv.dconv_causal(x, w, lengths=torch.zeros(2, dtype=torch.int32))),
        (dconv.DconvError, lambda: dconv.dconv_causal(x[:, :0], w)),
        (dconv.DconvError, lambda: dconv.dconv_causal(x, dev(8, 9))),
        (ValueError, lambda: dconv.dconv_causal_grad(x[:, :8], x, w)),
        (ValueError, lambda: dconv.dconv_causal_step(x[:, 0], dev(1, 3, 8), w)),               # fewer windows than rows
        (ValueError, lambda: dconv.dconv_causal_step(x[:, 0], dev(2, 4, 8), w)),
        (TypeError, lambda: dconv.dconv_causal_step(x[:, 0], dev(2, 3, 16)[:, :, ::2], w)),
    ]
    A, B = dev(8, 4, t=torch.float32), dev(2, 9, 2, 4)
    refused += [
        (TypeError, lambda: dconv.dconv_scan(x, x, dev(8, 4), B, B)),                          # A in 16 bits
        (TypeError, lambda: dconv.dconv_scan(x, x.float(), A, B, B)),
        (ValueError, lambda: dconv.dconv_scan(x, x, dev(7, 4, t=torch.float32), B, B)),
        (ValueError, lambda: dconv.dconv_scan(x, x, A, B[:, :, :, :3], B)),
        (ValueError, lambda: dconv.dconv_scan(x, x, A, B[:, :, 0], B)),
        (dconv.DconvError, lambda: dconv.dconv_scan(x, x, A, dev(2, 9, 3, 4), dev(2, 9, 3, 4))),   # 8 channels in 3 groups
        (dconv.DconvError, lambda: dconv.dconv_scan(x, x, dev(8, 33, t=torch.float32), dev(2, 9, 1, 33), dev(2, 9, 1, 33))),
        (TypeError, lambda: dconv.dconv_scan(x, x, A, B, B, state=dev(2, 8, 4))),
        (ValueError, lambda: dconv.dconv_scan(x, x, A, B, B, starts=dev(1, t=torch.float32))),
        (ValueError, lambda: dconv.dconv_scan_grad(x, x, x, A, B, B, z=dev(2, 9, 7))),
        (ValueError, lambda: dconv.dconv_scan_step(x[:, 0], x[:, 0], A, B[:, 0], B[:, 0], dev(1, 8, 4, t=torch.float32))),
        (TypeError, lambda: dconv.dconv_scan_step(x[:, 0], x[:, 0], A, B[:, 0], B[:, 0], dev(2, 8, 4))),
    ]
    for k, (error, call) in enumerate(refused):
        with pytest.raises(error):
            call()
            pytest.fail(f"call {k} was taken")


def test_the_structs_of_each_form_lay_their_fields_where_the_full_ones_have_them():
    sizes = ["dtype", "N", "L", "C", "F", "M", "silu", "reserved"]
    rows = lambda *names, fields=("p", "sn", "sl"): [f"{n}.{f}" for n in names for f in fields]
    forms = [
        (q._CAUSAL_PROMPT, rows("x", "out") + ["filt", "bias", "state", "state_out", "lengths"]),
        (q._CAUSAL_GRAD, rows("x", "dout", "dx") + ["filt", "bias", "state", "dstate_out", "dstate", "dfilt", "dbias", "lengths",
                                                    "workspace", "workspace_bytes"]),
        (q._CAUSAL_STEP, rows("x", "out", fields=("p", "sn")) + ["filt", "bias", "state_out", "slots"])]
    for form, names in forms:
        names = sizes + names
        v = list(range(1, len(names) + 1))
        assert form.pack(*v) == _pack(CAUSAL, q._CAUSAL, dict(zip(names, v)))
    sizes = ["dtype", "N", "L", "C", "S", "G", "M", "softplus"]
    group = ("p", "sn", "sl", "sg")
    forms = [
        (q._SCAN_PROMPT, rows("u", "delta", "z", "out") + rows("B", "Cm", fields=group) +
         ["A", "D", "delta_bias", "state", "state_out", "starts", "lengths", "workspace", "workspace_bytes"]),
        (q._SCAN_GRAD, rows("u", "delta", "z") + rows("B", "Cm", fields=group) + rows("dout", "du", "ddelta", "dz") +
         rows("dB", "dC", fields=group) + ["A", "D", "delta_bias", "state", "dstate_out", "dstate", "dA", "dD", "ddelta_bias",
                                           "starts", "lengths", "workspace", "workspace_bytes"]),
        (q._SCAN_STEP, rows("u", "delta", "z", "out", fields=("p", "sn")) + rows("B", "Cm", fields=("p", "sn", "sg")) +
         ["A", "D", "delta_bias", "state_out", "slots"])]
    for form, names in forms:
        names = sizes + names
        v = list(range(1, len(names) + 1))
        assert form.pack(*v) == _pack(SCAN, q._SCAN, dict(zip(names, v)))
