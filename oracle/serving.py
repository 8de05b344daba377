"""Plain statements of the serving operators in fp64: attention over packed prompts, single-token
attention behind a shared prefix, products with 4-bit weights.  Each function also returns what
its result's error is measured by: the sum of the magnitudes that were added up.

Pinned by tests/test_oracle_serving.py (closed forms, brute force)."""
import numpy as np


def _attend(q, k, v, scale):
    """One row against the tokens it may see: (output, sum of p |v| / sum of p)."""
    if k.shape[0] == 0:
        return np.zeros(v.shape[1]), np.zeros(v.shape[1])
    s = scale * (k @ q)
    p = np.exp(s - s.max())
    return (p @ v) / p.sum(), (p @ np.abs(v)) / p.sum()


def attn_prompt(q, k, v, edges, scale=None):
    """q [total, heads, dim]; k, v [total, kv_heads, dim]; edges: where the sequences begin and the last
    one ends.  Rows of no sequence are NaN."""
    total, heads, dim = q.shape
    group = heads // k.shape[1]
    scale = dim ** -0.5 if scale is None else scale
    out = np.full(q.shape, np.nan)
    mass = np.full(q.shape, np.nan)
    for a, b in zip(edges, edges[1:]):
        for i in range(a, b):
            for h in range(heads):
                out[i, h], mass[i, h] = _attend(q[i, h], k[a:i + 1, h // group], v[a:i + 1, h // group], scale)
    return out, mass


def attn_prefix(q, K, V, Ko, Vo, own_len, scale=None):
    """q [batch, heads, dim]; K, V [prefix, kv_heads, dim]; Ko, Vo [batch, own_cap, kv_heads, dim]."""
    batch, heads, dim = q.shape
    group = heads // K.shape[1]
    scale = dim ** -0.5 if scale is None else scale
    out, mass = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(batch):
        n = min(max(int(own_len[b]), 0), Ko.shape[1])
        for h in range(heads):
            g = h // group
            out[b, h], mass[b, h] = _attend(q[b, h], np.concatenate([K[:, g], Ko[b, :n, g]]),
                                            np.concatenate([V[:, g], Vo[b, :n, g]]), scale)
    return out, mass


def w4_codes(tiles, n, k):
    """Codes [n, k] from words [ceil(n/16), ceil(k/128), 64, 4]: word i of entry 16 q + r of tile (t, b) holds
    row 16 t + r, columns c = 128 b + 32 i + 8 q to c + 7, c + 2 j in bits 4 j, c + 2 j + 1 in bits 16 + 4 j."""
    words = np.asarray(tiles).astype(np.int64) & 0xFFFFFFFF
    codes = np.zeros((n, k), np.int64)
    row, col = np.arange(n)[:, None], np.arange(k)[None, :]
    b, rest = col // 128, col % 128
    i, q, e = rest // 32, rest % 32 // 8, rest % 8
    shift = 4 * (e // 2) + 16 * (e % 2)
    codes[:] = (words[row // 16, b, 16 * q + row % 16, i] >> shift) & 15
    return codes


def gemv_w4(x, codes, scales, zeros, group):
    """x [m, k], codes [n, k], scales and zeros [n, groups] (zeros None: 8).  The magnitudes are those of a
    sum of (128 + code) x and (128 + zero) x, scaled."""
    k = x.shape[1]
    g = np.arange(k) // group
    z = 8.0 if zeros is None else zeros[:, g].astype(np.float64)
    s = scales[:, g]
    return x @ ((codes - z) * s).T, np.abs(x) @ ((256.0 + codes + z) * np.abs(s)).T
