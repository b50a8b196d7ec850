"""The router's gradient keeps the 24 bits of dscores and its whole range.

A sum of two products, and zeros.  bf16: the three parts of a value hold it exactly and their products with a bf16 element are exact in
fp32, so six of them and what they are added to round fewer than 16 times, at most 2 u (u = 2^-24) of the absolute terms each."""
import numpy as np
import pytest

from oracle import block_ref as R
from tests.within import U, assert_within, dev

pytestmark = pytest.mark.gpu

SIZES = [(2, 8, 2), (40, 136, 2), (33, 256, 64), (70, 264, 130), (513, 1024, 70), (2050, 136, 12)]


def _run(T, d, nb, dtype, h, W, ds, check_dh, check_dW):
    import torch
    from paper_2406_04984_amd import binding as B
    s = B.make_shape(T, d, nb, 8, 1, 1, dtype)
    (ht, h), (wt, W), (dst, ds) = dev(h, dtype), dev(W, dtype), dev(ds, "f32")
    ws = torch.full((B.meft_block_workspace_bytes(s),), 0xFF, dtype=torch.uint8, device="cuda")
    dh, dW, db = torch.zeros_like(ht), torch.zeros_like(wt), torch.zeros((nb,), device="cuda")
    B.meft_route_bwd(s, ht, wt, dst, None, dh, dW, db, ws)
    dh_ref, dW_ref, _ = R.route_bwd(h, W, ds, None)
    if check_dh:
        assert_within("dh", dh, dh_ref, 32 * U * (np.abs(ds) @ np.abs(W)))
    if check_dW:
        assert_within("dWg", dW, dW_ref, 32 * U * (np.abs(ds).T @ np.abs(h)))


def _pair(r, n):
    """a, and -a without its last eight bits: their sum is a's last eight bits."""
    a = (r.uniform(1, 2, n) * np.exp2(r.randint(-20, 3, n)) * r.choice([-1, 1], n)).astype(np.float32)
    return a, -(a.view(np.uint32) & np.uint32(0xFFFFFF00)).view(np.float32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T, d, nb", SIZES)
def test_the_last_bits(T, d, nb, dtype):
    """Two equal rows times a value and its negative without the last bits: nothing but those is left."""
    r = np.random.RandomState(T + d + nb)
    h, W = r.standard_normal((T, d)), r.standard_normal((nb, d))
    W[1::2] = W[0:nb - nb % 2:2]
    ds = np.zeros((T, nb), np.float32)
    t, b = np.arange(T), 2 * r.randint(0, nb // 2, T)
    ds[t, b], ds[t, b + 1] = _pair(r, T)
    _run(T, d, nb, dtype, h, W, ds, True, False)
    h[1::2] = h[0:T - T % 2:2]
    ds = np.zeros((T, nb), np.float32)
    b, t = np.arange(nb), 2 * r.randint(0, T // 2, nb)
    ds[t, b], ds[t + 1, b] = _pair(r, nb)
    _run(T, d, nb, dtype, h, W, ds, False, True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T, d, nb", SIZES)
def test_values_beyond_the_largest_bf16(T, d, nb, dtype):
    """fp32 values that would round to an infinity in bf16 are numbers: so are their products with small elements."""
    r = np.random.RandomState(T * d + nb)
    h, W = 1e-3 * r.standard_normal((T, d)), 1e-3 * r.standard_normal((nb, d))
    ds = np.zeros((T, nb), np.float32)
    for i in range(min(T, nb)):          # one in a row and one in a column
        ds[i, i] = np.float32(r.choice([3.3962e38, 3.4e38, 3.4028234663852886e38]) * r.choice([-1, 1]))
    _run(T, d, nb, dtype, h, W, ds, True, True)
