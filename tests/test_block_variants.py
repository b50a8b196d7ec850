"""The GPU tests of norms and dropout reach every kernel of theirs that the library holds, so it holds none that no shape reaches.
Without a GPU: what the tests' sizes launch is recorded (tests/hip_recorder.c stands in for the HIP runtime)."""
import ctypes
import json
import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2406_04984_amd", "libmeft.so")
ARGS = {"norm_fwd": ["x", "gamma", "beta", "h", "mean", "rstd"],
        "norm_bwd": ["x", "gamma", "mean", "rstd", "dh", "dy", "dx", "dgamma", "dbeta"],
        "add_norm_fwd": ["step", "out", "res", "gamma", "beta", "y", "h", "mean", "rstd"],
        "add_norm_bwd": ["step", "y", "gamma", "mean", "rstd", "dh", "dy", "dres", "dout", "dgamma", "dbeta"],
        "dropout_add": ["step", "out", "res", "y"]}


def _main(rec_path):
    from tests.test_block_launches import _Drop, _Norm, _Rec, _Shape
    rec = ctypes.CDLL(rec_path, mode=ctypes.RTLD_GLOBAL)   # before the library: its symbols come first
    lib = ctypes.CDLL(LIB)
    rec.rec_at.restype = ctypes.POINTER(_Rec)
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    lib.meft_block_workspace_bytes.restype = sz
    names = set()
    for call, T, d, dtype, p, absent, in_place in json.load(sys.stdin):
        sp = ctypes.byref(_Shape(T, d, 32, 4, 8, 1, 1, dtype, 0, 0))
        at = {n: (i + 1) << 44 for i, n in enumerate(ARGS[call])}      # far apart
        at.update({out: at[place] for out, place in in_place.items()})
        at.update({n: None for n in absent})
        head = ([] if call == "dropout_add" else [ctypes.byref(_Norm(0, 1e-5))]) + (
            [] if call.startswith("norm") else [ctypes.byref(_Drop(p, 1, 2))])
        tail = [vp(1 << 50), sz(lib.meft_block_workspace_bytes(sp))] if call.endswith("bwd") else []
        rec.rec_clear()
        rc = getattr(lib, "meft_" + call)(sp, *head, *[vp(at[n]) for n in ARGS[call]], *tail, vp(None))
        assert rc == 0, (call, T, d, rc)
        names |= {rec.rec_at(i).contents.name.decode() for i in range(rec.rec_count())}
    print(json.dumps(sorted(names)))


def _sizes(test):
    """T and d of a parametrised test."""
    return next([v[:2] for v in m.args[1]] for m in test.pytestmark if m.name == "parametrize" and m.args[0].startswith("T, d"))


def _jobs():
    """The calls that the tests make."""
    from tests import test_gpu_block_rounds as rounds, test_gpu_dropout, test_gpu_norm
    none, gamma = ["dgamma", "dbeta"], ["dbeta"]
    for dt in (0, 1):
        for T, d in test_gpu_norm.SIZES + rounds.NORM:
            yield "norm_fwd", T, d, dt, 0, [], {}
            for absent, in_place in (([], {}), (none, {"dx": "dh"}), ([], {"dx": "dh"}), (gamma, {"dx": "dy"})):
                yield "norm_bwd", T, d, dt, 0, absent, in_place
        for p in (0, 0.1):
            for T, d in _sizes(test_gpu_norm.test_add_norm) + rounds.ADD_NORM:
                yield "add_norm_fwd", T, d, dt, p, [], {}
                for absent, in_place in (([], {}), (none, {"dres": "dy", "dout": "dh"}), ([], {"dres": "dh"}), ([], {"dout": "dh"})):
                    yield "add_norm_bwd", T, d, dt, p, absent, in_place
            for T, d in _sizes(rounds.test_add_norm_without_a_shift):
                yield "add_norm_bwd", T, d, dt, p, gamma, {}
        for T, d in _sizes(test_gpu_dropout.test_against_the_generator) + rounds.DROPOUT:
            for p in (0, 0.3):
                yield "dropout_add", T, d, dt, p, [], {}


@pytest.fixture(scope="module")
def launched(tmp_path_factory):
    rec = os.path.join(str(tmp_path_factory.mktemp("launches")), "hip_recorder.so")
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-O1", "-o", rec, os.path.join(ROOT, "tests", "hip_recorder.c"), "-ldl", "-pthread"])
    run = subprocess.run([sys.executable, "-m", "tests.test_block_variants", rec], input=json.dumps(list(_jobs())), text=True,
                         capture_output=True, timeout=300, cwd=ROOT)
    assert run.returncode == 0, run.stderr[-4000:]
    names = subprocess.run(["c++filt"], input="\n".join(json.loads(run.stdout)), text=True, capture_output=True, check=True).stdout
    return set(re.findall(r"meft::(?:__device_stub__)?(\w+<[^(\n]*>)\(", names))


@pytest.mark.parametrize("kernel", ["norm_fwd_kernel", "norm_bwd_kernel", "norm_grad_kernel", "dropout_add_kernel"])
def test_every_kernel_is_reached(kernel, launched):
    symbols = subprocess.check_output(["nm", "-C", LIB], text=True)
    have, reached = set(re.findall(r"__device_stub__(%s<[^(]*>)\(" % kernel, symbols)), {n for n in launched if n.startswith(kernel)}
    assert have and have == reached, (sorted(have - reached), sorted(reached - have))


if __name__ == "__main__":
    _main(sys.argv[1])
