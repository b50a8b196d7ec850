"""Infinities and NaN in the router's gradient: what they enter is infinite or NaN, everything else is as it is without them, bit
for bit."""
import numpy as np
import pytest

from tests.within import dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T, d, nb", [(5, 72, 3), (200, 264, 64), (530, 136, 130), (2050, 1024, 33)])
def test_it_stays_where_it_enters(T, d, nb, dtype, value):
    import torch
    from paper_2406_04984_amd import binding as B
    r = np.random.RandomState(T)
    s = B.make_shape(T, d, nb, 8, 1, 1, dtype)
    (h, _), (W, _), (add, _) = (dev(r.standard_normal(n), dtype) for n in ((T, d), (nb, d), (T, d)))
    ds, _ = dev(r.standard_normal((T, nb)), "f32")
    ds[T // 2] = 0                                    # a token that pads the batch
    ws = torch.empty((B.meft_block_workspace_bytes(s),), dtype=torch.uint8, device="cuda")

    def run(h, W, ds, add):
        dh, dW, db = torch.zeros_like(h), torch.zeros_like(W), torch.zeros((nb,), device="cuda")
        B.meft_route_bwd(s, h, W, ds, add, dh, dW, db, ws)
        return dh, dW, db

    good = run(h, W, ds, add)
    assert all(bool(x.isfinite().all()) for x in good)
    t, b, c = T - 1, nb - 1, d - 3

    def check(args, dh=(), dW=(), db=()):
        for got, want, place in zip(run(*args), good, (dh, dW, db)):
            off = torch.zeros_like(got, dtype=torch.bool)
            if place != ():
                off[place] = True
            assert bool((got.isfinite() != off).all()) and torch.equal(got[~off], want[~off])

    bad = ds.clone()
    bad[t, b] = value
    check((h, W, bad, add), dh=(t,), dW=(b,), db=(b,))
    bad = h.clone()
    bad[T // 2, c] = value                            # its dscores are 0 and it is no number all the same
    check((bad, W, ds, add), dW=(slice(None), c))
    bad = W.clone()
    bad[0, c] = value
    check((h, bad, ds, add), dh=(slice(None), c))
    bad = add.clone()
    bad[t, c] = value
    check((h, W, ds, bad), dh=(t, c))
