"""Plain 64-bit forms of the bounded-cache decoding operators, request by
request, and the batches that their tests run.  Imports nothing of the product."""
import numpy as np


def visible(j, k, window, n_sink):
    """Whether the row at position j sees the key at position k."""
    return (k <= j) & ((window == 0) | (j - k < window) | (k < n_sink))


def attention(q, k, v, ctx, window, n_sink, scale):
    """q [m, H, dh], k / v [ctx + m, KH, dh] float64 -> (o, a, n): the outputs
    [m, H, dh], the sums of softmax weights times |v| (the size of the terms
    that o is a sum of), and the keys that each row sees.  Keys that a row
    does not see take no part at all, whatever they hold."""
    m, H, dh = q.shape
    G = H // k.shape[1]
    o, a, n = np.zeros(q.shape), np.zeros(q.shape), np.zeros(m, np.int64)
    for i in range(m):
        see = visible(ctx + i, np.arange(ctx + m), window, n_sink)
        ks, vs = k[see], v[see]
        n[i] = see.sum()
        for h in range(H):
            s = ks[:, h // G] @ q[i, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            o[i, h] = p @ vs[:, h // G]
            a[i, h] = p @ np.abs(vs[:, h // G])
    return o, a, n


def score_sizes(q, k, scale):
    """[m, H]: the largest sum |q k| scale over the keys, the size of the terms of a row's scores."""
    G = q.shape[1] // k.shape[1]
    s = np.matmul(np.abs(q).transpose(1, 0, 2), np.abs(np.repeat(k, G, 1)).transpose(1, 2, 0))
    return s.max(-1).T * scale


def rotate(x, pos, theta):
    """Rotate-half of x [m, heads, dh] by positions pos, base theta (0: as it is)."""
    if theta == 0:
        return x.copy()
    half = x.shape[-1] // 2
    ang = pos[:, None].astype(np.float64) * np.exp(-np.log(np.float64(theta)) * np.arange(half) * 2.0 / x.shape[-1])
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * c - b * s, a * s + b * c], -1)


def sample(l, temperature, top_k, top_p, min_p, u):
    """(id, log probability, distance of u's target from the nearest border of
    the running sum, relative to the sum) of one request, fp64."""
    l = np.asarray(l, np.float64)
    ok = ~np.isnan(l)
    if not ok.any():
        return -1, np.nan, np.inf
    idx = np.nonzero(ok)[0]
    l = l[ok]
    by = np.lexsort((idx, -l))
    M = l[by[0]]
    if not temperature > 0:
        return int(idx[by[0]]), 0.0, np.inf
    T = min(max(float(temperature), 1e-30), 1e30)
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(l == M, 1.0, np.exp((l - M) / T))
    w = np.where(np.isnan(w), 0.0, w)
    ws = w[by]
    keep = np.ones(l.size, bool)
    if top_k > 0:
        keep[top_k:] = False
    c = np.cumsum(np.where(keep, ws, 0.0))
    if top_p < 1:
        keep &= c - ws < float(top_p) * c[-1]
    if min_p > 0:
        keep &= ws >= float(min_p)
    keep[0] = True
    kept = np.zeros(l.size, bool)
    kept[by[keep]] = True
    wk = np.where(kept, w, 0.0)
    c = np.cumsum(wk)
    target = (float(u) if u > 0 else 0.0) * c[-1]
    a = min(int(np.searchsorted(c, target, "right")), int(np.nonzero(wk > 0)[0][-1]))
    return int(idx[a]), float(np.log(wk[a] / c[-1])), float(np.abs(c - target).min() / c[-1])
