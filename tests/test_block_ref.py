"""The fp64 reference of the calls around the layer (oracle/block_ref.py) pinned: the generator's published answers, closed
forms, and every gradient against central differences."""
import numpy as np
import pytest

from oracle import block_ref as R


@pytest.mark.parametrize("counter, key, want", [
    ([0] * 4, [0, 0], [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]),
    ([0xffffffff] * 4, [0xffffffff] * 2, [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]),
    ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0], [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1])])
def test_generator(counter, key, want):
    got = R.philox([np.array([c], np.uint64) for c in counter], key)
    assert [int(g[0]) for g in got] == want


def test_mask_is_a_function_of_the_place():
    a, b = R.gain(40, 64, 0.3, 99, 7), R.gain(17, 40, 0.3, 99, 7)
    assert np.array_equal(a[:17, :40], b)
    for other in (R.gain(40, 64, 0.3, 98, 7), R.gain(40, 64, 0.3, 99, 8), R.gain(40, 64, 0.3, 99 + (1 << 32), 7),
                  R.gain(40, 64, 0.3, 99, 7 + (1 << 32))):
        assert 0.3 < (a != other).mean() < 0.55      # 2 * 0.3 * 0.7
    assert set(np.unique(R.gain(9, 64, 0.0, 1, 1))) == {1.0}
    g = R.gain(500, 1000, 0.1, 5, 6)
    assert abs((g == 0).mean() - 0.1) < 5 * np.sqrt(0.09 / 5e5) and abs(g.mean() - 1) < 0.01


def _diff(f, x, eps=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        old = x[i]
        x[i] = old + eps
        up = f()
        x[i] = old - eps
        g[i] = (up - f()) / (2 * eps)
        x[i] = old
    return g


@pytest.mark.parametrize("layer", [True, False])
def test_norm_gradient(layer):
    r = np.random.RandomState(3)
    x, gamma, beta, w, dy = r.randn(3, 8), r.randn(8), r.randn(8), r.randn(3, 8), r.randn(3, 8)

    def f():
        return float((R.norm_fwd(x, gamma, beta, layer, 1e-3)[0] * w).sum() + (x * dy).sum())

    _, mean, rstd = R.norm_fwd(x, gamma, beta, layer, 1e-3)
    dx, dgamma, dbeta = R.norm_bwd(x, gamma, mean, rstd, w, dy, layer)
    for got, at in ((dx, x), (dgamma, gamma), (dbeta, beta)):
        assert np.allclose(got, _diff(f, at), rtol=1e-6, atol=1e-7)


def test_balance_closed_forms():
    # even probabilities: L = 1 whatever the counts; one block takes all: L = B p
    idx = np.array([[0, 1], [2, 3], [0, 3]])
    counts, n, prob, loss = R.balance_fwd(np.zeros((3, 4)), idx, None, 2.0, 1.0)
    assert list(counts) == [2, 1, 1, 2] and n == 3 and np.allclose(prob, 0.75)
    assert np.isclose(loss[1], 1.0) and np.isclose(loss[2], np.log(4) ** 2) and np.isclose(loss[0], 2 + np.log(4) ** 2)
    s = np.tile([5.0, 0, 0, 0], (6, 1))
    loss = R.balance_fwd(s, np.zeros((6, 1), int), None, 1.0, 0.0)[3]
    assert np.isclose(loss[0], 4 * np.exp(5) / (np.exp(5) + 3))
    # nothing valid, nothing finite
    assert not R.balance_fwd(s, np.zeros((6, 1), int), np.zeros(6), 1.0, 1.0)[3].any()
    assert R.balance_fwd(np.full((6, 4), -np.inf), np.zeros((6, 1), int), None, 1.0, 1.0)[1] == 0


def test_balance_gradient():
    r = np.random.RandomState(4)
    s, idx, valid = r.randn(6, 5), r.randint(0, 5, (6, 2)), np.array([1, 1, 0, 1, 1, 1])
    s[1, 2] = -np.inf
    s[4] = -np.inf
    counts, n, _, _ = R.balance_fwd(s, idx, valid, 0.7, 0.3)
    got = R.balance_bwd(s, counts, n, 2, valid, 0.7, 0.3, 1.5)
    fin = np.isfinite(s)
    want = np.zeros_like(s)
    for i in np.argwhere(fin):
        i = tuple(i)
        old = s[i]
        f = []
        for h in (1e-6, -1e-6):
            s[i] = old + h
            f.append(R.balance_fwd(s, idx, valid, 0.7, 0.3)[3][0])
        s[i] = old
        want[i] = 1.5 * (f[0] - f[1]) / 2e-6
    assert np.allclose(got, want, rtol=1e-6, atol=1e-8) and n == 4
    assert not got[2].any() and not got[4].any() and got[1, 2] == 0


def test_ranks_add_up():
    """Counts and tokens summed over the ranks, then each rank's gradient: the whole batch's."""
    r = np.random.RandomState(5)
    s, idx = r.randn(12, 7), r.randint(0, 7, (12, 3))
    counts, n, _, _ = R.balance_fwd(s, idx, None, 1.0, 0.5)
    whole = R.balance_bwd(s, counts, n, 3, None, 1.0, 0.5, 1.0)
    parts = [R.balance_bwd(s[a:a + 4], counts, n, 3, None, 1.0, 0.5, 1.0) for a in (0, 4, 8)]
    assert np.allclose(np.concatenate(parts), whole, rtol=1e-12)


def test_route_gradient():
    r = np.random.RandomState(6)
    h, Wg, bias, ds, add = r.randn(5, 8), r.randn(3, 8), r.randn(3), r.randn(5, 3), r.randn(5, 8)

    def f():
        return float(((h @ Wg.T + bias) * ds).sum() + (h * add).sum())

    for got, at in zip(R.route_bwd(h, Wg, ds, add), (h, Wg, bias)):
        assert np.allclose(got, _diff(f, at), rtol=1e-6, atol=1e-7)
