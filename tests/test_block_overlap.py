"""Outputs that lie over operands which the backward calls around the layer go on reading are refused on the host; those that the
header allows are not.  Without a GPU: tests/hip_recorder.c stands in for the HIP runtime, so no launch follows an address here."""
import ctypes
import json
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2406_04984_amd", "libmeft.so")
D, NB = 64, 4
OK, INVALID = 0, 1
ARGS = {"norm_bwd": ["x", "gamma", "mean", "rstd", "dh", "dy", "dx", "dgamma", "dbeta"],
        "add_norm_bwd": ["y", "gamma", "mean", "rstd", "dh", "dy", "dres", "dout", "dgamma", "dbeta"],
        "route_bwd": ["h", "Wg", "dscores", "add", "dh", "dWg", "dbias"]}


def _main(rec_path):
    from tests.test_block_launches import _Drop, _Norm, _Shape
    rec = ctypes.CDLL(rec_path, mode=ctypes.RTLD_GLOBAL)   # before the library: its symbols come first
    lib = ctypes.CDLL(LIB)
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    lib.meft_block_workspace_bytes.restype = sz
    out = []
    for T, call, places in json.load(sys.stdin):
        sp = ctypes.byref(_Shape(T, D, NB * 8, NB, 8, 2, 1, 0, 0, 0))
        at = {n: (i + 1) << 40 for i, n in enumerate(ARGS[call])}      # far apart
        own = dict(at)
        rms = places.pop("rms", False)
        for n, where in places.items():
            at[n] = None if where is None else own[where[0]] + where[1]
        norm, drop = ctypes.byref(_Norm(int(rms), 1e-5)), ctypes.byref(_Drop(0.1, 1, 2))
        head = {"norm_bwd": (norm,), "add_norm_bwd": (norm, drop, vp(None)), "route_bwd": ()}[call]
        rec.rec_clear()
        rc = getattr(lib, "meft_" + call)(sp, *head, *[vp(at[n]) for n in ARGS[call]], vp(1 << 50),
                                          sz(lib.meft_block_workspace_bytes(sp)), vp(None))
        out.append([rc, rec.rec_count()])
    print(json.dumps(out))


def _results(jobs, tmp):
    rec = os.path.join(str(tmp), "hip_recorder.so")
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-O1", "-o", rec, os.path.join(ROOT, "tests", "hip_recorder.c"), "-ldl", "-pthread"])
    run = subprocess.run([sys.executable, "-m", "tests.test_block_overlap", rec], input=json.dumps(jobs), text=True, capture_output=True,
                         timeout=300, cwd=ROOT)
    assert run.returncode == 0, run.stderr[-4000:]
    return json.loads(run.stdout)


# T, call, {operand: (the operand that it lies over, bytes behind its start)}; fp32, so a row has 256 bytes
REFUSED = [
    (16, "norm_bwd", {"dx": ("x", 0)}), (1000, "norm_bwd", {"dx": ("x", 0)}), (16, "norm_bwd", {"dx": ("x", 0), "dgamma": None, "dbeta": None}),
    (16, "norm_bwd", {"dx": ("x", 256)}), (16, "norm_bwd", {"dx": ("x", 16 - 16 * 256)}), (16, "norm_bwd", {"dx": ("dh", 256)}),
    (16, "norm_bwd", {"dx": ("dy", -256)}), (16, "norm_bwd", {"dgamma": ("gamma", 0)}), (16, "norm_bwd", {"dbeta": ("gamma", 240)}),
    (16, "norm_bwd", {"dbeta": ("dgamma", 0)}), (16, "norm_bwd", {"dgamma": ("dx", 256)}), (16, "norm_bwd", {"dgamma": ("dh", 0)}),
    (16, "norm_bwd", {"dx": ("rstd", 48)}), (16, "norm_bwd", {"dx": ("mean", 48)}), (16, "add_norm_bwd", {"dres": ("y", 0)}), (16, "add_norm_bwd", {"dout": ("y", 15 * 256)}),
    (16, "add_norm_bwd", {"dout": ("dres", 256)}), (16, "add_norm_bwd", {"dout": ("dh", 512)}), (16, "add_norm_bwd", {"dgamma": ("gamma", 0)}),
    (16, "route_bwd", {"dh": ("h", 0)}), (16, "route_bwd", {"dh": ("h", 256), "add": None}), (16, "route_bwd", {"dh": ("add", 256)}),
    (16, "route_bwd", {"dh": ("dscores", 0)}), (16, "route_bwd", {"dh": ("Wg", 3 * 256)}), (16, "route_bwd", {"dWg": ("Wg", 0)}),
    (16, "route_bwd", {"dWg": ("h", 16)}), (16, "route_bwd", {"dWg": ("add", 0)}), (16, "route_bwd", {"dbias": ("dscores", 4)}),
    (16, "route_bwd", {"dWg": ("dh", 0)}), (0, "norm_bwd", {"dgamma": ("dbeta", 0)}),
]
ALLOWED = [
    (16, "norm_bwd", {}), (16, "norm_bwd", {"dx": ("dh", 0)}), (16, "norm_bwd", {"dx": ("dy", 0)}), (16, "norm_bwd", {"dh": ("x", 0), "dy": ("x", 0)}),
    (16, "norm_bwd", {"dx": ("x", 16 * 256)}), (16, "norm_bwd", {"dx": ("x", -16 * 256)}), (16, "norm_bwd", {"dgamma": ("gamma", 256)}),
    (16, "norm_bwd", {"dgamma": None, "dbeta": None, "dy": None}), (16, "norm_bwd", {"dy": ("dh", 0), "dx": ("dh", 0)}),
    (16, "add_norm_bwd", {}), (16, "add_norm_bwd", {"dres": ("dh", 0), "dout": ("dy", 0)}),
    (16, "add_norm_bwd", {"dres": ("dy", 0), "dout": ("dh", 0)}), (16, "route_bwd", {}), (16, "route_bwd", {"dh": ("add", 0)}),
    (16, "route_bwd", {"dh": ("h", 16 * 256)}), (16, "route_bwd", {"dWg": ("Wg", -4 * 256)}), (16, "route_bwd", {"dh": None, "add": None}),
    (16, "route_bwd", {"dWg": None, "dbias": None}),
    # the mean of the rms kind is not read
    (16, "norm_bwd", {"rms": True, "mean": ("dx", 0)}), (16, "add_norm_bwd", {"rms": True, "mean": ("dout", 64)}),
    # no token, no row that could be overwritten
    (0, "norm_bwd", {"dx": ("x", 0)}), (0, "add_norm_bwd", {"dres": ("y", 0)}), (0, "route_bwd", {"dh": ("h", 0)}),
]


@pytest.mark.parametrize("jobs, status", [(REFUSED, INVALID), (ALLOWED, OK)], ids=["refused", "allowed"])
def test_overlaps(jobs, status, tmp_path):
    for job, (rc, launches) in zip(jobs, _results(jobs, tmp_path)):
        assert rc == status and (launches > 0) == (status == OK), (job, rc, launches)


if __name__ == "__main__":
    _main(sys.argv[1])
