"""Norms on the GPU, forward, backward and fused with dropout and the residual add, against fp64.

Slack (u = 2^-24, the half step of fp32).  A sum over a row runs over at most 16 columns of a lane one after another, 6 steps
over a wave and 16 over the waves: fewer than 40 roundings, so mean is off by 40 u mean|x| and rstd by (40 + 40 mean|x| rstd + 4) u
relative; with A = 1 + mean|x| rstd, h is off by less than 64 u ((|xh| + 1) |gamma| A + |beta|).  Backward, with mean and rstd
given: xh is off by 3 u relative, the row's two means by 44 u of the mean absolute term, hence dx by less than
64 u (rstd (|g| + mean|g| + |xh| mean|g xh|) + |dy|).  dgamma and dbeta are sums over T tokens: (T + 32) u times the sum of
absolute terms."""
import numpy as np
import pytest

from oracle import block_ref as R
from tests.within import U, assert_guard, assert_within, dev, guarded, host64

pytestmark = pytest.mark.gpu
EPS = float(np.float32(1e-5))

SIZES = [(1, 4096), (3, 8), (5, 64), (37, 72), (130, 512), (33, 520), (1000, 768), (9, 1032), (21, 2048), (600, 4096), (7, 4104),
         (19, 8192), (3, 8200), (5, 16384)]


def _rows(r, T, d):
    """A stream whose channels differ, a few far larger, one row with a large mean, one constant but for a column."""
    x = r.standard_normal((T, d)) * r.uniform(0.25, 1.75, d) + 0.2 * r.standard_normal(d)
    x[:, r.randint(0, d, max(1, d // 100))] *= 8
    if T > 2:
        x[1] += 40
        x[2] = 0.5
        x[2, d // 2] = -3.0
    return x


def _fwd_slack(x, xh, rstd, gamma, beta):
    A = 1 + np.abs(x).mean(1, keepdims=True) * rstd[:, None]
    return 64 * U * ((np.abs(xh) + 1) * np.abs(gamma) * A + (0 if beta is None else np.abs(beta)))


def _stat_slack(x, rstd):
    A = np.abs(x).mean(1)
    return 40 * U * A, 64 * U * rstd * (1 + A * rstd)


def _bwd_slack(xh, g, rstd, dy):
    r = rstd[:, None]
    return 64 * U * (r * (np.abs(g) + np.abs(g).mean(1, keepdims=True) + np.abs(xh) * np.abs(g * xh).mean(1, keepdims=True)) + np.abs(dy))


def _shape(B, T, d, dtype):
    return B.make_shape(T, d, 4, 8, 1, 1, dtype)


def _f32(a):
    import torch
    return torch.from_numpy(np.asarray(a, np.float32)).cuda()


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T, d", SIZES)
def test_norm(T, d, dtype, kind):
    import torch
    from paper_2406_04984_amd import binding as B
    r = np.random.RandomState(T * 31 + d)
    layer, shift = kind == "layer", (kind == "layer") != (T % 2 == 0)
    s, hp = _shape(B, T, d, dtype), B.MeftNorm(B.MEFT_NORM_LAYER if layer else B.MEFT_NORM_RMS, EPS)
    (xt, x), (gt, gamma) = dev(_rows(r, T, d), dtype), dev(1 + 0.2 * r.standard_normal(d), dtype)
    (bt, beta) = dev(0.1 * r.standard_normal(d), dtype) if shift else (None, None)
    h_ref, mean, rstd = R.norm_fwd(x, gamma, beta, layer, EPS)
    whole, h = guarded((T, d), xt.dtype)
    mt, rt = torch.full((T + 1,), -7.0, device="cuda"), torch.full((T + 1,), -7.0, device="cuda")
    B.meft_norm_fwd(s, hp, xt, gt, bt, h, mt, rt)
    xh = (x - mean[:, None]) * rstd[:, None]
    assert_within("h", h, h_ref, _fwd_slack(x, xh, rstd, gamma, beta))
    ms, rs = _stat_slack(x, rstd)
    assert_within("mean", mt[:T], mean, ms)
    assert_within("rstd", rt[:T], rstd, rs)
    assert_guard(whole, T)
    assert float(mt[T]) == -7 and float(rt[T]) == -7
    # without the statistics, and over the input
    again = xt.clone()
    B.meft_norm_fwd(s, hp, again, gt, bt, again, None, None)
    assert torch.equal(again, h)

    # backward, on fp32 statistics that both sides are given
    mt, rt = _f32(mean), _f32(rstd)
    mean, rstd = host64(mt), host64(rt)
    (dht, dh), (dyt, dy) = dev(0.01 * r.standard_normal((T, d)), dtype), dev(0.01 * r.standard_normal((T, d)), dtype)
    ws = torch.full((B.meft_block_workspace_bytes(s),), 0xFF, dtype=torch.uint8, device="cuda")
    whole, dx = guarded((T, d), xt.dtype)
    wg, dgt = guarded((1, d), xt.dtype)
    wb, dbt = guarded((1, d), xt.dtype)
    B.meft_norm_bwd(s, hp, xt, gt, mt, rt, dht, dyt, dx, dgt, dbt, ws)
    dx_ref, dgamma, dbeta = R.norm_bwd(x, gamma, mean, rstd, dh, dy, layer)
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dh * gamma
    assert_within("dx", dx, dx_ref, _bwd_slack(xh, g, rstd, dy))
    assert_within("dgamma", dgt[0], dgamma, (T + 32) * U * np.abs(dh * xh).sum(0))
    assert_within("dbeta", dbt[0], dbeta, (T + 32) * U * np.abs(dh).sum(0))
    assert_guard(whole, T)
    assert_guard(wg, 1)
    assert_guard(wb, 1)
    # no gradient past the norm, frozen weights, in place of dh; only gamma's gradient; in place of dy
    want = dht.clone()
    B.meft_norm_bwd(s, hp, xt, gt, mt if layer else None, rt, want, None, want, None, None, ws)
    assert_within("dx", want, R.norm_bwd(x, gamma, mean, rstd, dh, None, layer)[0], _bwd_slack(xh, g, rstd, np.zeros_like(g)))
    over = dht.clone()
    dg3, db3 = torch.zeros_like(dgt), torch.zeros_like(dbt)
    B.meft_norm_bwd(s, hp, xt, gt, mt, rt, over, dyt, over, dg3, db3, ws)
    assert torch.equal(over, dx)
    assert_within("dgamma", dg3[0], dgamma, (T + 32) * U * np.abs(dh * xh).sum(0))
    assert_within("dbeta", db3[0], dbeta, (T + 32) * U * np.abs(dh).sum(0))
    dg2, inplace = torch.zeros_like(dgt), dyt.clone()
    B.meft_norm_bwd(s, hp, xt, gt, mt, rt, dht, inplace, inplace, dg2, None, ws)
    assert torch.equal(dg2, dgt) and torch.equal(inplace, dx)


@pytest.mark.parametrize("p", [0.0, 0.1, 0.9])
@pytest.mark.parametrize("dtype, kind", [("bf16", "rms"), ("bf16", "layer"), ("f32", "layer")])
@pytest.mark.parametrize("T, d", [(1, 4096), (5, 8), (37, 72), (333, 768), (70, 2048), (257, 4096), (11, 8200)])
def test_add_norm(T, d, dtype, kind, p):
    """One pass gives what the two calls give, and the gradients are the formula's; the stream it is the norm of is the stored one."""
    import torch
    from paper_2406_04984_amd import binding as B
    r = np.random.RandomState(T * 17 + d)
    layer = kind == "layer"
    s, hp = _shape(B, T, d, dtype), B.MeftNorm(B.MEFT_NORM_LAYER if layer else B.MEFT_NORM_RMS, EPS)
    seed, offset, count = 0x123456789ABCDEF0 + T, (1 << 64) - 3, 5          # the counter goes over the top of 64 bits
    drop = B.MeftDrop(p, seed, offset)
    step = torch.tensor([count], dtype=torch.int64, device="cuda")
    (xt, x), (ot, o) = dev(_rows(r, T, d), dtype), dev(0.3 * r.standard_normal((T, d)), dtype)
    (gt, gamma), (bt, beta) = dev(1 + 0.2 * r.standard_normal(d), dtype), dev(0.1 * r.standard_normal(d), dtype)
    wy, y = guarded((T, d), xt.dtype)
    wh, h = guarded((T, d), xt.dtype)
    mt, rt = torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
    B.meft_add_norm_fwd(s, hp, drop, step, ot, xt, gt, bt, y, h, mt, rt)
    gain = R.gain(T, d, p, seed, offset + count)
    assert_within("y", y, x + gain * o, 2 * U * (np.abs(x) + gain * np.abs(o)))
    ys = host64(y)
    h_ref, mean, rstd = R.norm_fwd(ys, gamma, beta, layer, EPS)
    assert_within("h", h, h_ref, _fwd_slack(ys, (ys - mean[:, None]) * rstd[:, None], rstd, gamma, beta))
    assert_guard(wy, T)
    assert_guard(wh, T)
    # the two calls; over the inputs
    y2, h2, m2, r2 = torch.zeros_like(y), torch.zeros_like(h), torch.zeros_like(mt), torch.zeros_like(rt)
    B.meft_dropout_add(s, drop, step, ot, xt, y2)
    B.meft_norm_fwd(s, hp, y2, gt, bt, h2, m2, r2)
    assert torch.equal(y2, y) and torch.equal(h2, h) and torch.equal(m2, mt) and torch.equal(r2, rt)
    o3, x3 = ot.clone(), xt.clone()
    B.meft_add_norm_fwd(s, hp, drop, step, o3, x3, gt, bt, x3, o3, None, None)
    assert torch.equal(x3, y) and torch.equal(o3, h)

    mean, rstd = host64(mt), host64(rt)
    (dht, dh), (dyt, dy) = dev(0.01 * r.standard_normal((T, d)), dtype), dev(0.01 * r.standard_normal((T, d)), dtype)
    ws = torch.full((B.meft_block_workspace_bytes(s),), 0xFF, dtype=torch.uint8, device="cuda")
    wr, dres = guarded((T, d), xt.dtype)
    wo, dout = guarded((T, d), xt.dtype)
    dg, db = torch.zeros_like(gt), torch.zeros_like(gt)
    B.meft_add_norm_bwd(s, hp, drop, step, y, gt, mt, rt, dht, dyt, dres, dout, dg, db, ws)
    dx_ref, dgamma, dbeta = R.norm_bwd(ys, gamma, mean, rstd, dh, dy, layer)
    xh, g = (ys - mean[:, None]) * rstd[:, None], dh * gamma
    slack = _bwd_slack(xh, g, rstd, dy)
    assert_within("dres", dres, dx_ref, slack)
    assert_within("dout", dout, gain * dx_ref, gain * (slack + 2 * U * np.abs(dx_ref)))
    assert_within("dgamma", dg, dgamma, (T + 32) * U * np.abs(dh * xh).sum(0))
    assert_within("dbeta", db, dbeta, (T + 32) * U * np.abs(dh).sum(0))
    assert_guard(wr, T)
    assert_guard(wo, T)
    a, b = dht.clone(), dyt.clone()
    B.meft_add_norm_bwd(s, hp, drop, step, y, gt, mt, rt, a, b, b, a, None, None, ws)
    assert torch.equal(b, dres) and torch.equal(a, dout)
    for one, two in ((0, 1), (1, 0)):       # dres or dout in place of dh, with the weights' gradients
        bufs = [dht.clone(), torch.zeros_like(dht)]
        B.meft_add_norm_bwd(s, hp, drop, step, y, gt, mt, rt, bufs[0], dyt, bufs[one], bufs[two], dg, db, ws)
        assert torch.equal(bufs[one], dres) and torch.equal(bufs[two], dout)
        assert_within("dgamma", dg, dgamma, (T + 32) * U * np.abs(dh * xh).sum(0))
        assert_within("dbeta", db, dbeta, (T + 32) * U * np.abs(dh).sum(0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_add_norm_without_dropout(dtype):
    """No dropout given (serving): the same as a share of 0, forward and backward."""
    import torch
    from paper_2406_04984_amd import binding as B
    T, d = 3, 4096
    r = np.random.RandomState(9)
    s, hp, none = _shape(B, T, d, dtype), B.MeftNorm(B.MEFT_NORM_RMS, EPS), B.MeftDrop(0.0, 5, 6)
    (x, _), (o, _), (g, _), (dh, _) = (dev(r.standard_normal(n), dtype) for n in ((T, d), (T, d), (d,), (T, d)))
    got = []
    for drop in (None, none):
        y, h, rs = torch.zeros_like(x), torch.zeros_like(x), torch.zeros(T, device="cuda")
        dres, dout, dg = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(g)
        ws = torch.empty((B.meft_block_workspace_bytes(s),), dtype=torch.uint8, device="cuda")
        B.meft_add_norm_fwd(s, hp, drop, None, o, x, g, None, y, h, None, rs)
        B.meft_add_norm_bwd(s, hp, drop, None, y, g, None, rs, dh, None, dres, dout, dg, None, ws)
        assert torch.equal(dres, dout) and bool(dres.any())
        got.append((y, h, rs, dres, dg))
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_a_row_that_is_no_number_stays_alone():
    import torch
    from paper_2406_04984_amd import binding as B
    T, d = 12, 768
    s, hp = _shape(B, T, d, "bf16"), B.MeftNorm(B.MEFT_NORM_LAYER, EPS)
    xt, _ = dev(np.random.RandomState(1).standard_normal((T, d)), "bf16")
    gt, _ = dev(np.ones(d), "bf16")
    good, h = torch.zeros_like(xt), torch.zeros_like(xt)
    B.meft_norm_fwd(s, hp, xt, gt, None, good, None, None)
    xt[3, 5], xt[7, 9] = float("nan"), float("inf")
    B.meft_norm_fwd(s, hp, xt, gt, None, h, None, None)
    assert bool(h[3].isnan().all()) and bool(h[7].isnan().any())
    rest = [i for i in range(T) if i not in (3, 7)]
    assert torch.equal(h[rest], good[rest])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_tokens(dtype):
    import torch
    from paper_2406_04984_amd import binding as B
    s, hp = _shape(B, 0, 520, dtype), B.MeftNorm(B.MEFT_NORM_LAYER, EPS)
    some, _ = dev(np.ones((1, 520)), dtype)
    f, dg, db = torch.ones(4, device="cuda"), some[0].clone(), some[0].clone()
    ws = torch.full((B.meft_block_workspace_bytes(s),), 0xFF, dtype=torch.uint8, device="cuda")
    B.meft_norm_bwd(s, hp, some, some, f, f, some, None, some, dg, db, ws)
    assert not dg.any() and not db.any() and bool((some == 1).all())


def test_same_bits_every_time():
    import torch
    from paper_2406_04984_amd import binding as B
    T, d = 3001, 1024
    s, hp = _shape(B, T, d, "f32"), B.MeftNorm(B.MEFT_NORM_LAYER, EPS)
    r = np.random.RandomState(2)
    (x, _), (dh, _), (g, _) = (dev(r.standard_normal(n), "f32") for n in ((T, d), (T, d), (d,)))
    h, m, rs, dx = torch.zeros_like(x), torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda"), torch.zeros_like(x)
    B.meft_norm_fwd(s, hp, x, g, None, h, m, rs)
    got = []
    for fill in (0x00, 0xFF, 0x7F):
        ws = torch.full((B.meft_block_workspace_bytes(s),), fill, dtype=torch.uint8, device="cuda")
        dg, db = torch.zeros_like(g), torch.zeros_like(g)
        B.meft_norm_bwd(s, hp, x, g, m, rs, dh, None, dx, dg, db, ws)
        got.append((dg, db))
    assert all(torch.equal(a, b) for k in got[1:] for a, b in zip(k, got[0]))
