"""The 4-bit prefix cache and tree attention over it from their definitions, in 64 bits (numpy), for the tests."""
import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def encode_block(x):
    """(codes [32], scale byte) of one block by search: the smallest e with max|x| <= 7 2^e, the nearest magnitude, ties to the even code."""
    x = np.asarray(x, np.float64)
    if not np.isfinite(x).all():
        return np.zeros(32, np.uint8), 255
    amax, e = np.abs(x).max(), -119
    while e < 125 and amax > 7.0 * 2.0 ** e:
        e += 1
    y = x / 2.0 ** e
    dist = np.abs(np.abs(y)[:, None] - MAGNITUDES[None])
    code = np.empty(32, np.uint8)
    for i in range(32):
        best = dist[i].min()
        ties = np.flatnonzero(dist[i] == best)
        code[i] = min(ties, key=lambda c: (c % 2, c))
    return (code + 8 * np.signbit(y)).astype(np.uint8), e + 127


def encode(rows):
    """codes uint8 [..., d/32, 32] and scales uint8 [..., d/32] of rows [..., d], vectorised."""
    x = np.asarray(rows, np.float64)
    x = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    bad = ~np.isfinite(x).all(-1)
    y = np.where(bad[..., None], 0.0, x)
    amax = np.abs(y).max(-1)
    e = np.full(amax.shape, -119.0)
    while True:
        up = (amax > 7.0 * 2.0 ** e) & (e < 125)
        if not up.any():
            break
        e = e + up
    y = y / 2.0 ** e[..., None]
    a = np.abs(y)
    mid = (MAGNITUDES[1:] + MAGNITUDES[:-1]) / 2
    code = np.zeros(a.shape, np.uint8)
    for c in range(7):          # past the middle, or on it where the upper code is the even one
        code += ((a > mid[c]) | ((a == mid[c]) & (c % 2 == 1))).astype(np.uint8)
    code = np.where(bad[..., None], 0, code + 8 * np.signbit(y)).astype(np.uint8)
    return code, np.where(bad, 255, e + 127).astype(np.uint8)


def decode(codes, scales):
    """Rows float64 [..., d]."""
    v = MAGNITUDES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    factor = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127.0))
    with np.errstate(invalid="ignore"):
        v = v * factor[..., None]
    return v.reshape(*codes.shape[:-2], -1)


def pool_rows(codes, scales):
    """Logical rows float64 [n_pages][H_kv][page_size][d] of pools in the library's layout."""
    lo, hi = codes & 15, codes >> 4
    c = np.stack((lo, hi), -1).reshape(*codes.shape[:-1], 32)             # [P][H][tiles][nb][16][32]
    c, s = np.moveaxis(c, -3, -2), np.moveaxis(scales, -2, -1)            # [P][H][tiles][16][nb][32]
    rows = decode(c, s)
    return rows.reshape(*rows.shape[:-3], -1, rows.shape[-1])


def ancestors(parent):
    n = len(parent)
    vis = np.zeros((n, n), bool)
    for i in range(n):
        a = i
        while a >= 0:
            vis[i, a] = True
            a = parent[a]
    return vis


def attention(q, k, v, k_tree, v_tree, vis, scale):
    """One sequence: q [N][H_q][d], k/v [H_kv][L][d], k/v_tree [H_kv][N][d], vis [N][N] (row sees column), all float64.
    Returns out [N][H_q][d] and a bound on what rounding may take from it, derived as follows.  With weights p_j (sum 1):
      the weights enter PV as bf16, at most 2^-8 of each: sum p_j |v_j| 2^-8;
      the output is rounded to bf16: |out| 2^-8 (and 2^-134 where it is subnormal);
      a score is a sum of d products in fp32, off by at most (d + 2) 2^-24 sum |q k| scale, then multiplied by scale log2(e) and
      taken from the maximum in fp32: another 4 2^-24 (|s| + |max|), which scales a weight by as much; exp2 and the
      sums of weights and of PV (L + N terms in fp32, at most a few thousand partial sums deep) 2^-14 of the weight."""
    N, H_q, d = q.shape
    G = H_q // k.shape[0]
    L = k.shape[1]
    out, bound = np.empty_like(q), np.empty_like(q)
    for h in range(H_q):
        g = h // G
        kk, vv = np.concatenate((k[g], k_tree[g])), np.concatenate((v[g], v_tree[g]))
        s = q[:, h] @ kk.T * scale
        mag = np.abs(q[:, h]) @ np.abs(kk).T * scale
        s[:, L:][~vis] = -np.inf
        top = s.max(-1, keepdims=True)
        with np.errstate(invalid="ignore"):
            p = np.exp(s - top)
        p /= p.sum(-1, keepdims=True)
        ds = 2.0 ** -24 * ((d + 2) * mag + 4 * (np.where(np.isfinite(s), np.abs(s), 0) + np.abs(top)))
        rel = 2.0 ** -8 + 2.0 ** -14 + 2 * (ds + ds.max(-1, keepdims=True))
        out[:, h] = p @ vv
        bound[:, h] = (p * rel) @ np.abs(vv) + np.abs(out[:, h]) * (2.0 ** -8 + (p * ds).sum(-1, keepdims=True) * 2) + 2.0 ** -134
    return out, bound
