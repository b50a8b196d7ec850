"""The calls around the layer in numpy fp64, from their formulas (include/meft.h): norms, dropout and its generator, the
router's balance loss, and their gradients.  Shares nothing with the HIP path.  Test infrastructure only."""
import numpy as np

_LOW = np.uint64(0xFFFFFFFF)


def philox(counter, key):
    """Philox4x32, 10 rounds: counter (4 arrays of uint64 holding 32-bit words), key (2 words) -> 4 arrays."""
    x = [np.asarray(c, np.uint64) & _LOW for c in counter]
    k = [int(key[0]), int(key[1])]
    for _ in range(10):
        p0, p1 = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        hi0, lo0, hi1, lo1 = p0 >> np.uint64(32), p0 & _LOW, p1 >> np.uint64(32), p1 & _LOW
        x = [hi1 ^ x[1] ^ np.uint64(k[0]), lo1, hi0 ^ x[3] ^ np.uint64(k[1]), lo0]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return x


def threshold(p):
    return int(np.floor(float(np.float32(p)) * 65536.0 + 0.5))


def gain(T, d, p, seed, offset):
    """[T, d]: 0 where an element goes, else 65536 / (65536 - threshold)."""
    thr = threshold(p)
    offset %= 1 << 64
    c, t = np.meshgrid(np.arange((d + 7) // 8, dtype=np.uint64), np.arange(T, dtype=np.uint64))
    words = philox([c, t, np.full_like(c, offset & 0xFFFFFFFF), np.full_like(c, offset >> 32)],
                   [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF])
    u16 = np.empty((T, c.shape[1], 8), np.int64)
    for w in range(4):
        u16[:, :, 2 * w] = (words[w] & np.uint64(0xFFFF)).astype(np.int64)
        u16[:, :, 2 * w + 1] = (words[w] >> np.uint64(16)).astype(np.int64)
    return np.where(u16.reshape(T, -1)[:, :d] >= thr, 65536.0 / (65536.0 - thr), 0.0)


def norm_fwd(x, gamma, beta, layer, eps):
    """h, mean, rstd"""
    mean = x.mean(axis=1) if layer else np.zeros(x.shape[0])
    xc = x - mean[:, None]
    rstd = 1.0 / np.sqrt((xc * xc).mean(axis=1) + eps)
    h = xc * rstd[:, None] * gamma
    return h + beta if beta is not None else h, mean, rstd


def norm_bwd(x, gamma, mean, rstd, dh, dy, layer):
    """dx, dgamma, dbeta"""
    xh, g = (x - mean[:, None]) * rstd[:, None], dh * gamma
    dx = g - xh * (g * xh).mean(axis=1, keepdims=True)
    if layer:
        dx = dx - g.mean(axis=1, keepdims=True)
    dx = dx * rstd[:, None]
    return dx + dy if dy is not None else dx, (dh * xh).sum(axis=0), dh.sum(axis=0)


def _softmax(scores, valid):
    """P, lse and which tokens count"""
    T = scores.shape[0]
    on = np.ones(T, bool) if valid is None else valid.astype(bool)
    on = on & ~np.all(scores == -np.inf, axis=1)
    P, lse = np.zeros_like(scores), np.zeros(T)
    for t in np.nonzero(on)[0]:
        m = scores[t].max()
        ex = np.exp(scores[t] - m)
        P[t], lse[t] = ex / ex.sum(), m + np.log(ex.sum())
    return P, lse, on


def balance_fwd(scores, block_idx, valid, w_balance, w_z):
    """counts, n, prob, (loss, L, Z)"""
    B, e = scores.shape[1], block_idx.shape[1]
    P, lse, on = _softmax(scores, valid)
    picked = block_idx[on].ravel()
    counts = np.bincount(picked[(picked >= 0) & (picked < B)], minlength=B)
    n, prob = int(on.sum()), P.sum(axis=0)
    if n == 0:
        return counts, 0, prob, np.zeros(3)
    L, Z = B * float((counts * prob).sum()) / (n * n * e), float((lse * lse)[on].sum()) / n
    return counts, n, prob, np.array([(w_balance * L if w_balance else 0.0) + (w_z * Z if w_z else 0.0), L, Z])


def balance_bwd(scores, counts, n, e, valid, w_balance, w_z, dloss):
    B = scores.shape[1]
    P, lse, on = _softmax(scores, valid)
    if n == 0:
        return np.zeros_like(scores)
    f = counts / (n * e)
    ds = P * (w_balance * B / n * (f - (P * f).sum(axis=1, keepdims=True)) + 2 * w_z / n * lse[:, None])
    return dloss * ds * on[:, None]


def route_bwd(h, Wg, ds, add):
    """dh, dWg, dbias"""
    dh = ds @ Wg
    return dh + add if add is not None else dh, ds.T @ h, ds.sum(axis=0)
