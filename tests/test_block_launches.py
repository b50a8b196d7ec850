"""What the calls around the layer ask of the HIP runtime, without a GPU (tests/hip_recorder.c stands in for it): launches within
the hardware's limits over the whole range of shapes, all on the caller's stream, and nothing but launches; and that the shapes of
the GPU tests reach every variant of the kernels."""
import ctypes
import json
import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2406_04984_amd", "libmeft.so")
STREAM = 0x77
CALLS = ["norm_fwd", "norm_bwd", "dropout_add", "add_norm_fwd", "add_norm_bwd", "route_scores", "balance_fwd", "balance_bwd", "route_bwd"]


class _Shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "d", "N", "n_blocks", "block_size", "top_e", "top_k", "dtype",
                                              "activation")] + [("flags", ctypes.c_uint32)]


class _Rec(ctypes.Structure):
    _fields_ = [("what", ctypes.c_char * 8), ("name", ctypes.c_char * 256), ("grid", ctypes.c_uint32 * 3),
                ("block", ctypes.c_uint32 * 3), ("lds", ctypes.c_uint64), ("stream", ctypes.c_uint64),
                ("event", ctypes.c_uint64), ("dst", ctypes.c_uint64), ("src", ctypes.c_uint64),
                ("bytes", ctypes.c_uint64)]


class _Norm(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("eps", ctypes.c_float)]


class _Drop(ctypes.Structure):
    _fields_ = [("p", ctypes.c_float), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64)]


class _Balance(ctypes.Structure):
    _fields_ = [("balance", ctypes.c_float), ("z", ctypes.c_float)]


def _main(rec_path):
    rec = ctypes.CDLL(rec_path, mode=ctypes.RTLD_GLOBAL)   # before the library: its symbols come first
    lib = ctypes.CDLL(LIB)
    rec.rec_at.restype = ctypes.POINTER(_Rec)
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    lib.meft_workspace_bytes.restype = lib.meft_block_workspace_bytes.restype = sz
    out = []
    for (T, d, nb, e, dtype), call, p in json.load(sys.stdin):
        s = _Shape(T, d, nb * 8, nb, 8, e, 1, dtype, 0, 0)
        sp = ctypes.byref(s)
        at = [vp((i + 1) << 44) for i in range(16)]   # one address per operand, far apart
        norm, drop, bal = ctypes.byref(_Norm(0, 1e-5)), ctypes.byref(_Drop(p, 1, 2)), ctypes.byref(_Balance(1, 1))
        ws = (at[15], sz((lib.meft_workspace_bytes if call == "route_scores" else lib.meft_block_workspace_bytes)(sp)))
        assert ws[1].value > 0, (T, d, nb, e)
        head, n, tail = {"norm_fwd": ((norm,), 6, ()), "norm_bwd": ((norm,), 9, ws), "dropout_add": ((drop,), 4, ()),
                         "add_norm_fwd": ((norm, drop), 9, ()), "add_norm_bwd": ((norm, drop), 11, ws), "route_scores": ((), 6, ws),
                         "balance_fwd": ((bal,), 7, ws), "balance_bwd": ((bal,), 6, ()), "route_bwd": ((), 7, ws)}[call]
        rec.rec_clear()
        rc = getattr(lib, "meft_" + call)(sp, *head, *at[:n], *tail, vp(STREAM))
        assert rc == 0, (call, rc)
        rows = []
        for i in range(rec.rec_count()):
            r = rec.rec_at(i).contents
            rows.append(dict(what=r.what.decode(), name=r.name.decode(), grid=list(r.grid), block=list(r.block), lds=r.lds,
                             stream=r.stream))
        out.append(rows)
    print(json.dumps(out))


def record(jobs, tmp):
    rec = os.path.join(str(tmp), "hip_recorder.so")
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-O1", "-o", rec, os.path.join(ROOT, "tests", "hip_recorder.c"), "-ldl", "-pthread"])
    run = subprocess.run([sys.executable, os.path.abspath(__file__), rec], input=json.dumps(jobs), text=True, capture_output=True, timeout=300)
    assert run.returncode == 0, run.stderr[-4000:]
    return json.loads(run.stdout)


SHAPES = [(1, 8, 1, 1), (1, 4096, 64, 4), (7, 72, 3, 2), (1000, 768, 32, 4), (8192, 4096, 64, 4), (4096, 4096, 256, 8),
          (16384, 1024, 256, 8), (513, 2048, 1024, 8), (100, 8192, 1025, 3), (64, 8200, 5000, 4), (33, 16384, 16384, 2),
          (300000, 16384, 16, 1), (1 << 21, 8192, 128, 1), ((1 << 28) - 1, 8, 2, 1), (40, 16384, 1, 1)]


@pytest.mark.parametrize("call", CALLS)
def test_launches(call, tmp_path):
    # the selection, meft_route's own, takes a wave a token: up to 2^26 tokens
    jobs = [[[*s, dt], call, 0.25] for s in SHAPES for dt in (0, 1) if call != "route_scores" or s[0] < 1 << 26]
    for (shape, _, _), rows in zip(jobs, record(jobs, tmp_path)):
        assert rows and {r["what"] for r in rows} == {"launch"}, (shape, rows)
        for r in rows:
            assert r["stream"] == STREAM and r["name"], (shape, r)
            threads = r["block"][0] * r["block"][1] * r["block"][2]
            assert 64 <= threads <= 1024 and threads % 64 == 0, (shape, r)
            assert all(g >= 1 for g in r["grid"]) and r["grid"][0] * r["block"][0] < 1 << 32, (shape, r)
            assert r["grid"][1] <= 65535 and r["grid"][2] <= 65535, (shape, r)
            assert r["lds"] <= 160 << 10, (shape, r)


def test_no_tokens(tmp_path):
    """Sums over tokens are written (zeros); what else there is launches nothing."""
    got = record([[[0, 72, 5, 2, dt], call, 0.25] for call in CALLS for dt in (0, 1)], tmp_path)
    wrote = {c: bool(got[2 * i]) and bool(got[2 * i + 1]) for i, c in enumerate(CALLS)}
    assert {c for c, w in wrote.items() if w} == {"norm_bwd", "add_norm_bwd", "balance_fwd", "route_bwd"}


def _variants(rows):
    return {re.sub(r"^_ZN?\d*meft\d*", "", r["name"]) for r in rows}


def test_gpu_tests_reach_every_variant(tmp_path):
    """The kernels that the tests' shapes launch, against all that the library holds of them."""
    from tests import test_gpu_balance, test_gpu_norm, test_gpu_route_grad
    jobs = [[[T, d, 4, 1, dt], "norm_fwd", 0] for T, d in test_gpu_norm.SIZES for dt in (0, 1)]
    jobs += [[[T, 64, nb, e, 0], c, 0] for T, nb, e in test_gpu_balance.SIZES for c in ("balance_fwd", "balance_bwd")]
    jobs += [[[T, d, nb, 1, dt], "route_bwd", 0] for T, d, nb in test_gpu_route_grad.SIZES for dt in (0, 1)]
    names = set().union(*map(_variants, record(jobs, tmp_path)))
    symbols = subprocess.check_output(["nm", "-C", LIB], text=True)
    for kernel, keep in (("norm_fwd_kernel", r", 0>"), ("balance_part_kernel", ""), ("balance_grad_kernel", ""), ("route_grad_kernel", ""),
                         ("route_dw_join_kernel", "")):
        have = set(re.findall(r"__device_stub__(%s<[^(]*>)\(" % kernel, symbols))
        have = {h for h in have if not keep or re.search(keep, h)}
        reached = {n for n in names if kernel in n}
        assert have and len(reached) == len(have), (kernel, sorted(have), sorted(reached))


if __name__ == "__main__":
    _main(sys.argv[1])
