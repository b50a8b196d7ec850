"""What the calls around the layer refuse, on the host: every call here is rejected before a device is touched."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x1000          # never followed on the host


@pytest.fixture(scope="module")
def B():
    if not os.path.exists(os.path.join(ROOT, "paper_2406_04984_amd", "libmeft.so")):
        import __graft_entry__
        __graft_entry__.build()
    from paper_2406_04984_amd import binding
    return binding


def _shape(B, **kw):
    base = dict(T=16, d=64, n_blocks=4, block_size=8, top_e=2, top_k=4, dtype="f32")
    base.update(kw)
    return B.make_shape(**base)


NAN, INF = float("nan"), float("inf")


def _calls(B):
    """name -> (its arguments with made-up addresses, the bad ones of each place, and whether the last two are a workspace)"""
    need = B.meft_block_workspace_bytes(_shape(B))
    norm, drop, bal = B.MeftNorm(0, 1e-5), B.MeftDrop(0.1, 1, 2), B.MeftBalance(1.0, 0.0)
    norms = [None, B.MeftNorm(2, 1e-5), B.MeftNorm(-1, 1e-5), B.MeftNorm(0, -1.0), B.MeftNorm(0, NAN), B.MeftNorm(1, INF)]
    drops = [B.MeftDrop(p, 0, 0) for p in (-0.1, 1.0, 0.999995, NAN, INF)]
    bals = [None, B.MeftBalance(NAN, 0), B.MeftBalance(1, INF)]
    must, may, four, byte = [None, P + 8], [P + 8], [None, P + 2], []
    maybe4 = [P + 2]
    return {
        "meft_norm_fwd": ([norm, P, P, P, P, P, P], [norms, must, must, may, must, maybe4, maybe4], False),
        "meft_norm_bwd": ([norm, P, P, P, P, P, P, P, P, P, P, need],
                          [norms, must, must, four, four, must, may, must, may + [None], may, None, None], True),
        "meft_dropout_add": ([drop, P, P, P, P], [drops, [P + 4], must, may, must], False),
        "meft_add_norm_fwd": ([norm, drop, P, P, P, P, P, P, 2 * P, P, P],
                              [norms, drops, [P + 4], must, must, must, may, must + [2 * P], must, maybe4, maybe4], False),
        "meft_add_norm_bwd": ([norm, drop, P, P, P, P, P, P, P, P, 2 * P, P, P, P, need],
                              [norms, drops, [P + 4], must, must, four, four, must, may, must + [2 * P], must, may + [None], may,
                               None, None], True),
        "meft_route_scores": ([P, P, P, P, P, P, P, B.meft_workspace_bytes(_shape(B))],
                              [must, must, byte, [None], byte, must, None, None], True),
        "meft_balance_fwd": ([bal, P, P, P, P, P, P, P, P, need], [bals, must, four, byte, four, four, four, four, None, None], True),
        "meft_balance_bwd": ([bal, P, P, P, P, P, P], [bals, must, four, four, byte, maybe4, must], False),
        "meft_route_bwd": ([P, P, P, P, P, P, P, P, need], [must, must, must, may, must, may, maybe4, None, None], True),
    }


NAMES = ["meft_norm_fwd", "meft_norm_bwd", "meft_dropout_add", "meft_add_norm_fwd", "meft_add_norm_bwd", "meft_route_scores",
         "meft_balance_fwd", "meft_balance_bwd", "meft_route_bwd"]


def _call(B, name, shape, args):
    args = [ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args]
    return getattr(B._lib, name)(ctypes.byref(shape) if shape is not None else None, *args, None)


@pytest.mark.parametrize("name", NAMES)
def test_refusals(B, name):
    good, bad, has_ws = _calls(B)[name]
    assert len(good) == len(bad)
    shape = _shape(B)
    for i, values in enumerate(bad):
        for v in values or []:
            args = list(good)
            args[i] = v
            assert _call(B, name, shape, args) == B.MEFT_ERR_INVALID_ARG, (i, v)
    if has_ws:
        for ws, n in ((None, 0), (None, good[-1]), (P + 16, good[-1]), (P, good[-1] - 1)):
            assert _call(B, name, shape, good[:-2] + [ws, n]) == B.MEFT_ERR_WORKSPACE
    assert _call(B, name, None, good) == B.MEFT_ERR_INVALID_ARG
    assert _call(B, name, _shape(B, top_e=9), good) == B.MEFT_ERR_INVALID_ARG
    assert _call(B, name, _shape(B, d=60), good) == B.MEFT_ERR_UNSUPPORTED
    assert _call(B, name, _shape(B, d=16392), good) == B.MEFT_ERR_UNSUPPORTED


def test_norms_of_the_rms_kind_need_no_mean(B):
    good = _calls(B)["meft_norm_bwd"][0]
    rms = [B.MeftNorm(1, 1e-5)] + good[1:]
    rms[3] = None
    assert _call(B, "meft_norm_bwd", _shape(B), rms[:-1] + [0]) == B.MEFT_ERR_WORKSPACE      # past the pointers' checks


def test_route_bwd_needs_an_output(B):
    good = _calls(B)["meft_route_bwd"][0]
    args = list(good)
    args[3:7] = [None] * 4
    assert _call(B, "meft_route_bwd", _shape(B), args) == B.MEFT_ERR_INVALID_ARG


def test_no_tokens(B):
    """T == 0: what has nothing to write returns at once (no device here, so a launch would fail)."""
    s = _shape(B, T=0)
    for name in ("meft_norm_fwd", "meft_dropout_add", "meft_add_norm_fwd", "meft_route_scores", "meft_balance_bwd"):
        good = _calls(B)[name][0]
        if name == "meft_route_scores":
            good = good[:-1] + [B.meft_workspace_bytes(s)]
        assert _call(B, name, s, good) == B.MEFT_OK, name


def test_workspace(B):
    assert B.meft_block_workspace_bytes(_shape(B, top_e=9)) == 0
    assert B.meft_block_workspace_bytes(_shape(B, T=0)) >= 256
    big = _shape(B, T=8192, d=4096, n_blocks=64, block_size=1024, top_e=4, top_k=256, dtype="bf16")
    assert 256 <= B.meft_block_workspace_bytes(big) < 64 << 20
    assert ctypes.sizeof(B.MeftDrop) == 24 and ctypes.sizeof(B.MeftNorm) == 8 and ctypes.sizeof(B.MeftBalance) == 8
