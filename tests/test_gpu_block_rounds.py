"""The calls around the layer at sizes where a workgroup walks several rounds of rows, holds several rows at once, or stores past
L2: the checks of the calls' own tests, against fp64, at the sizes below.  (tests/test_block_variants.py: these and the other sizes
reach every kernel.)"""
import numpy as np
import pytest

from oracle import block_ref as R
from tests import test_gpu_balance, test_gpu_dropout, test_gpu_norm
from tests.within import U, assert_within, dev, host64

pytestmark = pytest.mark.gpu

# two rounds and more forward (4096 rows of up to 1024 columns, 1024 of up to 2048, 512 beyond) and backward; two rows of a workgroup
NORM = [(4501, 72), (4501, 1000), (700, 768), (1100, 2048), (1100, 4096), (600, 5000), (530, 16384)]
PAST = [(16400, 1024), (4100, 4096)]       # 32 MB and more of bf16


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T, d", NORM)
def test_norm(T, d, dtype, kind):
    test_gpu_norm.test_norm(T, d, dtype, kind)


@pytest.mark.parametrize("T, d", PAST)
def test_norm_past_l2(T, d):
    test_gpu_norm.test_norm(T, d, "bf16", "layer" if d < 2048 else "rms")


# rows of few tokens as well, of the widths that the calls' own test leaves out
ADD_NORM = NORM + [(5, 5000), (3, 8192)]


@pytest.mark.parametrize("p", [0.0, 0.1])
@pytest.mark.parametrize("dtype, kind", [("bf16", "rms"), ("bf16", "layer"), ("f32", "rms")])
@pytest.mark.parametrize("T, d", ADD_NORM)
def test_add_norm(T, d, dtype, kind, p):
    test_gpu_norm.test_add_norm(T, d, dtype, kind, p)


@pytest.mark.parametrize("p", [0.0, 0.1])
@pytest.mark.parametrize("dtype, kind", [("bf16", "rms"), ("f32", "layer")])
@pytest.mark.parametrize("T, d", ADD_NORM)
def test_add_norm_without_a_shift(T, d, dtype, kind, p):
    """No beta: dgamma alone.  The slacks are those of the norms' tests."""
    import torch
    from paper_2406_04984_amd import binding as B
    r = np.random.RandomState(T * 13 + d)
    layer = kind == "layer"
    s, hp = test_gpu_norm._shape(B, T, d, dtype), B.MeftNorm(B.MEFT_NORM_LAYER if layer else B.MEFT_NORM_RMS, test_gpu_norm.EPS)
    drop = B.MeftDrop(p, 99, T)
    (xt, x), (ot, o) = dev(test_gpu_norm._rows(r, T, d), dtype), dev(0.3 * r.standard_normal((T, d)), dtype)
    (gt, gamma), (dht, dh) = dev(1 + 0.2 * r.standard_normal(d), dtype), dev(0.01 * r.standard_normal((T, d)), dtype)
    y, h, mt, rt = torch.zeros_like(xt), torch.zeros_like(xt), torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
    B.meft_add_norm_fwd(s, hp, drop, None, ot, xt, gt, None, y, h, mt, rt)
    gain = R.gain(T, d, p, 99, T)
    assert_within("y", y, x + gain * o, 2 * U * (np.abs(x) + gain * np.abs(o)))
    ys, mean, rstd = host64(y), host64(mt), host64(rt)
    h_ref, m_ref, r_ref = R.norm_fwd(ys, gamma, None, layer, test_gpu_norm.EPS)
    assert_within("h", h, h_ref, test_gpu_norm._fwd_slack(ys, (ys - m_ref[:, None]) * r_ref[:, None], r_ref, gamma, None))
    ws = torch.full((B.meft_block_workspace_bytes(s),), 0xFF, dtype=torch.uint8, device="cuda")
    dres, dout, dg = torch.zeros_like(y), torch.zeros_like(y), torch.zeros_like(gt)
    B.meft_add_norm_bwd(s, hp, drop, None, y, gt, mt, rt, dht, None, dres, dout, dg, None, ws)
    dx_ref, dgamma, _ = R.norm_bwd(ys, gamma, mean, rstd, dh, None, layer)
    xh, g = (ys - mean[:, None]) * rstd[:, None], dh * gamma
    slack = test_gpu_norm._bwd_slack(xh, g, rstd, np.zeros_like(g))
    assert_within("dres", dres, dx_ref, slack)
    assert_within("dout", dout, gain * dx_ref, gain * (slack + 2 * U * np.abs(dx_ref)))
    assert_within("dgamma", dg, dgamma, (T + 32) * U * np.abs(dh * xh).sum(0))


# a round is 524288 groups of eight columns: two to five rounds, rows that do not divide it
DROPOUT = [(4300, 1000), (130000, 72), (16800, 1000)]      # the last one past L2 in bf16


@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T, d", DROPOUT)
def test_dropout(T, d, p, dtype):
    test_gpu_dropout.test_against_the_generator(T, d, p, dtype)


# forward a round is 4096 rows of up to 256 blocks, 2048 of up to 1024, 256 beyond; backward 8192 and 2048
BALANCE = [(9001, 64, 4), (8500, 100, 3), (9001, 256, 8), (8300, 500, 4), (8200, 1000, 2), (2100, 1100, 3), (2100, 2500, 5), (2060, 4097, 2)]


@pytest.mark.parametrize("kind", ["all", "padded", "shut"])
@pytest.mark.parametrize("T, nb, e", BALANCE)
def test_balance(T, nb, e, kind):
    test_gpu_balance.test_against_fp64(T, nb, e, kind)
