"""The router's gradient, and the scores that meft_route_scores hands out, against fp64.

Slack (u = 2^-24).  fp32: products and sums over n terms, (n + 32) 2 u times the sum of absolute products.  bf16: dscores in two
bf16 parts keeps it to 2^-8 of 2^-8 (half a step of each part): 2^-16 relative, on top of the same sums."""
import numpy as np
import pytest

from oracle import block_ref as R
from paper_2406_04984_amd import synth
from tests.within import U, assert_guard, assert_within, dev, guarded, host64

pytestmark = pytest.mark.gpu

SIZES = [(1, 8, 1), (1, 4096, 64), (3, 72, 5), (16, 128, 32), (17, 136, 33), (64, 64, 64), (65, 120, 65), (1000, 768, 32),
         (777, 1000, 64), (300, 264, 130), (255, 512, 256), (70, 384, 300), (33, 256, 1030), (2049, 2048, 48), (513, 4096, 100), (40, 264, 640), (5000, 1024, 602)]


def _slack(dtype, terms, n):
    return ((2.0 ** -16 if dtype == "bf16" else 0) + 2 * U * (n + 32)) * terms


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T, d, nb", SIZES)
def test_gradient(T, d, nb, dtype):
    import torch
    from paper_2406_04984_amd import binding as B
    r = np.random.RandomState(T + d + nb)
    s = B.make_shape(T, d, nb, 8, 1, 1, dtype)
    (ht, h), (wt, W), (at, add) = (dev(x, dtype) for x in (
        r.standard_normal((T, d)), r.standard_normal((nb, d)) / np.sqrt(d), 0.01 * r.standard_normal((T, d))))
    ds = r.standard_normal((T, nb)) * np.exp(r.uniform(-8, 0, (T, nb)))
    ds[r.randint(T)] = 0
    dst, ds = dev(ds, "f32")
    ws = torch.full((B.meft_block_workspace_bytes(s),), 0xFF, dtype=torch.uint8, device="cuda")
    (w1, dh), (w2, dW), (w3, db) = guarded((T, d), ht.dtype), guarded((nb, d), ht.dtype), guarded((nb,), torch.float32)
    B.meft_route_bwd(s, ht, wt, dst, at, dh, dW, db, ws)
    dh_ref, dW_ref, db_ref = R.route_bwd(h, W, ds, add)
    a = np.abs(ds)
    dh_slack, dW_slack = _slack(dtype, a @ np.abs(W), nb) + 2 * U * np.abs(add), _slack(dtype, a.T @ np.abs(h), T)
    assert_within("dh", dh, dh_ref, dh_slack)
    assert_within("dWg", dW, dW_ref, dW_slack)
    assert_within("dbias", db, db_ref, (T + 32) * U * a.sum(0))
    for w, n in ((w1, T), (w2, nb), (w3, nb)):
        assert_guard(w, n)
    # no other gradient of h; in its place; each output alone
    alone = torch.zeros_like(dh)
    B.meft_route_bwd(s, ht, wt, dst, None, alone, None, None, ws)
    assert_within("dh", alone, ds @ W, _slack(dtype, a @ np.abs(W), nb))
    inplace = at.clone()
    B.meft_route_bwd(s, ht, wt, dst, inplace, inplace, None, None, ws)
    assert torch.equal(inplace, dh)
    W2, b2 = torch.zeros_like(dW), torch.zeros_like(db)
    ws.fill_(0x7F)
    B.meft_route_bwd(s, ht, wt, dst, None, None, W2, None, ws)
    B.meft_route_bwd(s, ht, wt, dst, None, None, None, b2, ws)
    assert torch.equal(W2, dW) and torch.equal(b2, db)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_tokens(dtype):
    import torch
    from paper_2406_04984_amd import binding as B
    s = B.make_shape(0, 72, 5, 8, 1, 1, dtype)
    some, _ = dev(np.ones((5, 72)), dtype)
    dW, db = some.clone(), torch.ones(5, device="cuda")
    ws = torch.full((B.meft_block_workspace_bytes(s),), 0xFF, dtype=torch.uint8, device="cuda")
    B.meft_route_bwd(s, some, some, torch.ones((1, 5), device="cuda"), None, some, dW, db, ws)
    assert not dW.any() and not db.any() and bool((some == 1).all())


@pytest.mark.parametrize("kw", [
    dict(T=5, d=64, n_blocks=4, block_size=16, top_e=2, top_k=8, dtype="bf16"),
    dict(T=300, d=256, n_blocks=64, block_size=16, top_e=4, top_k=8, dtype="bf16"),
    dict(T=5000, d=256, n_blocks=64, block_size=16, top_e=4, top_k=8, dtype="bf16"),      # contraction on tiles
    dict(T=77, d=72, n_blocks=100, block_size=8, top_e=3, top_k=4, dtype="f32"),
    dict(T=130, d=64, n_blocks=200, block_size=8, top_e=3, top_k=4, dtype="f32"),
    dict(T=130, d=64, n_blocks=700, block_size=8, top_e=9, top_k=4, dtype="bf16"),        # keys in registers
    dict(T=130, d=64, n_blocks=700, block_size=8, top_e=3, top_k=4, dtype="bf16"),        # keys in LDS
], ids=lambda kw: f"{kw['T']}x{kw['n_blocks']}-{kw['dtype']}")
@pytest.mark.parametrize("bias", [False, True])
def test_scores(kw, bias):
    """The same choice and scores as meft_route's, bit for bit, and all scores: the chosen ones' values stand in them, and they
    are the products in fp64 up to 2 (d + 32) u of the absolute ones."""
    import torch
    from paper_2406_04984_amd import binding as B
    from paper_2406_04984_amd.harness import DeviceLayer
    t = synth.make_inputs(synth.small_case(seed=77, **kw))
    if bias:
        t.bias = np.linspace(-0.5, 0.5, kw["n_blocks"]).astype(np.float32)
    la = DeviceLayer(t)
    la.route()
    want_idx, want_score = la.block_idx.clone(), la.block_score.clone()
    la.block_idx.fill_(-1)
    la.block_score.fill_(float("nan"))
    whole, scores = guarded((kw["T"], kw["n_blocks"]), torch.float32)
    B.meft_route_scores(la.shape, la.h, la.Wg, la.bias, la.block_idx, la.block_score, scores, la.ws)
    assert torch.equal(la.block_idx, want_idx) and torch.equal(la.block_score, want_score)
    assert torch.equal(scores.gather(1, want_idx.long()), want_score)
    assert_guard(whole, kw["T"])
    h, W = host64(la.h), host64(la.Wg)
    b = 0 if t.bias is None else t.bias.astype(np.float64)
    assert_within("scores", scores, h @ W.T + b, 2 * (kw["d"] + 32) * U * (np.abs(h) @ np.abs(W).T + np.abs(b)))
