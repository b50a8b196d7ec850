"""Operands past 4 GB: zeros but for the last tokens, whose rows have to come out as those of a small call with them alone.  Where
the kernels share out tokens differently the sums may round differently: their slack is that of the tests of the calls."""
import numpy as np
import pytest

from oracle import block_ref as R
from tests.within import U, assert_within, dev, host64

pytestmark = pytest.mark.gpu

T, D, N = (1 << 19) + 37, 4104, 70       # 4.3 GB of bf16; the last N tokens hold something


def _tail(x):
    import torch
    whole = torch.zeros((T, *x.shape[1:]), dtype=x.dtype, device="cuda")
    whole[-N:] = x
    return whole


def test_norm():
    import torch
    from paper_2406_04984_amd import binding as B
    r = np.random.RandomState(1)
    big, small = B.make_shape(T, D, 4, 8, 1, 1, "bf16"), B.make_shape(N, D, 4, 8, 1, 1, "bf16")
    hp = B.MeftNorm(B.MEFT_NORM_LAYER, 1e-5)
    (x, xs), (dh, dhs), (g, gs) = (dev(r.standard_normal(n), "bf16") for n in ((N, D), (N, D), (D,)))
    h, m, rs = torch.zeros_like(x), torch.zeros(N, device="cuda"), torch.zeros(N, device="cuda")
    B.meft_norm_fwd(small, hp, x, g, None, h, m, rs)
    dx = torch.zeros_like(x)
    ws = torch.empty((B.meft_block_workspace_bytes(big),), dtype=torch.uint8, device="cuda")
    B.meft_norm_bwd(small, hp, x, g, m, rs, dh, None, dx, None, None, ws)
    X = _tail(x)
    M, Rs = torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
    B.meft_norm_fwd(big, hp, X, g, None, X, M, Rs)           # in place
    assert torch.equal(X[-N:], h) and torch.equal(M[-N:], m) and torch.equal(Rs[-N:], rs) and not X[:-N].any()
    X.zero_()
    X[-N:] = x
    DH = _tail(dh)
    dg, db = torch.zeros_like(g), torch.zeros_like(g)
    B.meft_norm_bwd(big, hp, X, g, M, Rs, DH, None, DH, dg, db, ws)
    assert torch.equal(DH[-N:], dx) and not DH[:-N].any()
    xh = (xs - host64(m)[:, None]) * host64(rs)[:, None]
    assert_within("dgamma", dg, (dhs * xh).sum(0), (N + 64) * U * np.abs(dhs * xh).sum(0))
    assert_within("dbeta", db, dhs.sum(0), (N + 64) * U * np.abs(dhs).sum(0))


def test_router_gradient():
    import torch
    from paper_2406_04984_amd import binding as B
    r = np.random.RandomState(2)
    nb = 20
    big = B.make_shape(T, D, nb, 8, 1, 1, "bf16")
    (h, hs), (add, adds), (W, Ws) = (dev(r.standard_normal(n), "bf16") for n in ((N, D), (N, D), (nb, D)))
    ds, dss = dev(r.standard_normal((N, nb)), "f32")
    ws = torch.empty((B.meft_block_workspace_bytes(big),), dtype=torch.uint8, device="cuda")
    H, A, S = _tail(h), _tail(add), _tail(ds)
    dW, db = torch.zeros_like(W), torch.zeros(nb, device="cuda")
    B.meft_route_bwd(big, H, W, S, A, A, dW, db, ws)
    dh_ref, dW_ref, db_ref = R.route_bwd(hs, Ws, dss, adds)
    a = np.abs(dss)
    assert_within("dh", A[-N:], dh_ref, (2.0 ** -16 + 2 * U * (nb + 32)) * (a @ np.abs(Ws)) + 2 * U * np.abs(adds))
    assert not A[:-N].any()
    assert_within("dWg", dW, dW_ref, (2.0 ** -16 + 2 * U * (N + 32)) * (a.T @ np.abs(hs)))
    assert_within("dbias", db, db_ref, (N + 32) * U * a.sum(0))
