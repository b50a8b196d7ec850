"""The balance loss, its counts and its gradient against fp64; whole numbers are compared exactly.

Slack (u = 2^-24).  P = exp(x - top) / sum: x - top is off by u |x - top|, exp and the division by a few u more, the sum by at
most 40 u (16 scores of a lane, 6 steps over a wave, 16 waves): 64 u (1 + range) relative, range = top - lowest finite score that
matters (exp(-100) = 0).  lse is off by 64 u (1 + |lse|).  Sums over T tokens add (T + 32) u times the sum of absolute terms."""
import numpy as np
import pytest

from oracle import block_ref as R
from tests.within import U, assert_guard, assert_within, guarded, host64

pytestmark = pytest.mark.gpu

SIZES = [(1, 1, 1), (1, 64, 4), (3, 5, 2), (64, 64, 4), (777, 64, 4), (130, 100, 3), (2048, 256, 8), (50, 300, 5), (37, 1000, 16), (20, 1000, 100),
         (33, 1024, 2), (41, 1025, 3), (20, 2048, 8), (6, 3000, 5), (9, 4097, 2), (300, 5000, 4), (5, 16384, 300), (4000, 7, 7)]


def _inputs(T, nb, e, kind):
    r = np.random.RandomState(T + 7 * nb + e)
    s = r.standard_normal((T, nb)) * 2 - 1.1 * np.log(r.permutation(nb) + 1.0)
    idx = np.argsort(-s, axis=1, kind="stable")[:, :e].astype(np.int32)
    valid = None
    if kind != "all":
        valid = np.where(r.uniform(size=T) < 0.6, r.choice([1, 2, 255], T), 0).astype(np.uint8)
        s[valid == 0] = np.nan                                  # what pads the batch is not looked at
        idx[valid == 0] = 10 ** 9
    if kind == "shut" and nb > 1:
        s[:, r.randint(nb)] = -np.inf                           # a block that nobody may take
        s[r.randint(T)] = -np.inf                               # a token that has no block
        s[r.randint(T)] = -3.4028234663852886e38                # a row of the type's lowest value
        idx[r.randint(T), 0] = -1
        idx[r.randint(T), e - 1] = nb
    return s.astype(np.float32), idx, valid


@pytest.mark.parametrize("kind", ["all", "padded", "shut"])
@pytest.mark.parametrize("T, nb, e", SIZES)
def test_against_fp64(T, nb, e, kind):
    import torch
    from paper_2406_04984_amd import binding as B
    s32, idx, valid = _inputs(T, nb, e, kind)
    shape = B.make_shape(T, 64, nb, 8, e, 1, "bf16")
    z_weight = 0.0 if kind == "shut" else 0.25                  # the square of the lowest value is beyond fp32
    hp = B.MeftBalance(0.5, z_weight)
    st, it = torch.from_numpy(s32).cuda(), torch.from_numpy(idx).cuda()
    vt = None if valid is None else torch.from_numpy(valid).cuda()
    (wc, counts), (wn, n), (wp, prob), (wl, loss) = (guarded((k,), t) for k, t in (
        (nb, torch.int32), (1, torch.int32), (nb, torch.float32), (3, torch.float32)))
    ws = torch.full((B.meft_block_workspace_bytes(shape),), 0xFF, dtype=torch.uint8, device="cuda")
    B.meft_balance_fwd(shape, hp, st, it, vt, counts, n, prob, loss, ws)
    s = s32.astype(np.float64)
    s[np.isnan(s)] = 0
    c_ref, n_ref, p_ref, l_ref = R.balance_fwd(s, idx, valid, 0.5, z_weight)
    assert np.array_equal(counts.cpu().numpy(), c_ref) and int(n) == n_ref
    P, lse, on = R._softmax(s, valid)
    finite = np.where(np.isfinite(s), s, s.max(1, keepdims=True))
    rel = 64 * U * (1 + np.minimum(100, s.max(1, initial=-1e30) - finite.min(1)))[:, None]
    p_slack = (P * rel).sum(0) + (T + 32) * U * p_ref
    assert_within("prob", prob, p_ref, p_slack)
    if n_ref:
        scale = nb / (n_ref * n_ref * e)
        l_slack = scale * ((c_ref * p_slack).sum() + 64 * U * (c_ref * p_ref).sum())
        z_ref = l_ref[2]
        dl = 64 * U * (1 + np.abs(lse))
        z_slack = (2 * np.abs(lse) * dl + dl * dl)[on].sum() / n_ref + (T + 32) * U * z_ref
        assert_within("L", loss[1:2], l_ref[1:2], l_slack)
        if kind != "shut":
            assert_within("Z", loss[2:3], l_ref[2:3], z_slack)
        assert_within("loss", loss[:1], l_ref[:1], 0.5 * l_slack + (z_weight * z_slack if z_weight else 0) + 4 * U * abs(l_ref[0]))
    else:
        assert not loss.any()
    for w, k in ((wc, nb), (wn, 1), (wp, nb), (wl, 3)):
        assert_guard(w, k)

    dloss = torch.tensor([1.5], device="cuda")
    whole, ds = guarded((T, nb), torch.float32)
    B.meft_balance_bwd(shape, hp, st, counts, n, vt, dloss, ds)
    ref = R.balance_bwd(s, c_ref, n_ref, e, valid, 0.5, z_weight, 1.5)
    if n_ref:
        f = c_ref / (n_ref * e)
        a, b = 1.5 * 0.5 * nb / n_ref, 1.5 * 2 * z_weight / n_ref
        mean = (P * f).sum(1, keepdims=True)
        slack = P * (rel * (a * (f + mean) + b * np.abs(lse)[:, None]) + a * mean * rel + b * 64 * U * (1 + np.abs(lse))[:, None])
        assert_within("dscores", ds, ref * on[:, None], (slack + 64 * U * np.abs(ref)) * on[:, None])
    else:
        assert not ds.any()
    assert_guard(whole, T)
    # dloss 1 by default; in place of the scores
    one, inplace = torch.zeros_like(ds), st.clone()
    B.meft_balance_bwd(shape, hp, st, counts, n, vt, torch.ones(1, device="cuda"), one)
    B.meft_balance_bwd(shape, hp, inplace, counts, n, vt, None, inplace)
    assert torch.equal(one, inplace)


def test_nothing_valid_and_no_tokens():
    import torch
    from paper_2406_04984_amd import binding as B
    for T, nb in ((5, 64), (0, 64), (3, 2000), (0, 3)):
        shape, hp = B.make_shape(T, 64, nb, 8, 2, 1, "f32"), B.MeftBalance(1.0, 1.0)
        st = torch.full((max(T, 1), nb), float("nan"), device="cuda")
        it = torch.zeros((max(T, 1), 2), dtype=torch.int32, device="cuda")
        counts, n = torch.full((nb,), 9, dtype=torch.int32, device="cuda"), torch.full((1,), 9, dtype=torch.int32, device="cuda")
        prob, loss = torch.full((nb,), 9.0, device="cuda"), torch.full((3,), 9.0, device="cuda")
        ws = torch.full((B.meft_block_workspace_bytes(shape),), 0xFF, dtype=torch.uint8, device="cuda")
        vt = torch.zeros((max(T, 1),), dtype=torch.uint8, device="cuda")
        B.meft_balance_fwd(shape, hp, st, it, vt, counts, n, prob, loss, ws)
        assert not counts.any() and not n.any() and not prob.any() and not loss.any()
        ds = torch.full_like(st, 9.0)
        B.meft_balance_bwd(shape, hp, st, counts, n, vt, None, ds)
        assert not ds[:T].any()


def test_a_score_that_is_no_number_shows():
    """In a valid row it reaches the loss and the row's gradient, and no other row's."""
    import torch
    from paper_2406_04984_amd import binding as B
    T, nb = 40, 64
    shape, hp = B.make_shape(T, 64, nb, 8, 2, 1, "f32"), B.MeftBalance(1.0, 0.1)
    for value in (float("nan"), float("inf")):
        for everywhere in (False, True):
            st = torch.randn((T, nb), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
            st[7, (slice(None) if everywhere else 3)] = value
            it = torch.zeros((T, 2), dtype=torch.int32, device="cuda")
            counts, n = torch.zeros((nb,), dtype=torch.int32, device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda")
            prob, loss, ds = torch.zeros((nb,), device="cuda"), torch.zeros((3,), device="cuda"), torch.zeros_like(st)
            ws = torch.empty((B.meft_block_workspace_bytes(shape),), dtype=torch.uint8, device="cuda")
            B.meft_balance_fwd(shape, hp, st, it, None, counts, n, prob, loss, ws)
            B.meft_balance_bwd(shape, hp, st, counts, n, None, None, ds)
            assert int(n) == T and bool(loss[:2].isnan().all())
            rows = ds.isnan().any(1)
            assert bool(rows[7]) and int(rows.sum()) == 1


def test_ranks_add_up():
    """Two ranks' counts and tokens added up before the backward: the gradients are the whole batch's."""
    import torch
    from paper_2406_04984_amd import binding as B
    T, nb, e = 96, 32, 4
    s32, idx, valid = _inputs(T, nb, e, "padded")
    hp = B.MeftBalance(0.7, 0.2)

    def fwd(a, b):
        shape = B.make_shape(b - a, 64, nb, 8, e, 1, "f32")
        st, it, vt = (torch.from_numpy(np.ascontiguousarray(x[a:b])).cuda() for x in (s32, idx, valid))
        counts, n = torch.zeros((nb,), dtype=torch.int32, device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda")
        ws = torch.empty((B.meft_block_workspace_bytes(shape),), dtype=torch.uint8, device="cuda")
        B.meft_balance_fwd(shape, hp, st, it, vt, counts, n, torch.zeros(nb, device="cuda"), torch.zeros(3, device="cuda"), ws)
        return shape, st, vt, counts, n

    whole, parts = fwd(0, T), [fwd(0, 37), fwd(37, T)]
    counts, n = parts[0][3] + parts[1][3], parts[0][4] + parts[1][4]
    assert torch.equal(counts, whole[3]) and torch.equal(n, whole[4])
    got = []
    for shape, st, vt, c, k in parts + [whole]:
        ds = torch.zeros_like(st)
        B.meft_balance_bwd(shape, hp, st, counts, n, vt, None, ds)
        got.append(ds)
    assert torch.equal(torch.cat(got[:2]), got[2]) and bool(host64(got[2]).any())
