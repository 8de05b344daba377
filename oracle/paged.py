"""Plain statements in fp64 of rotary positions, of appending to the paged 8-bit cache and of single-token
attention over it.

Pinned by tests/test_oracle_paged.py (closed forms, brute force)."""
import numpy as np

from .serving import _attend


def rope(x, positions, freqs, interleaved=False, inverse=False, magnitude=1.0):
    """x [tokens, heads, dim]; returns the turned x and, per element, the magnitudes that were added up."""
    out, mass = np.array(x, dtype=np.float64), np.abs(x).astype(np.float64)
    n = len(freqs)
    a = np.asarray(positions, np.float64)[:, None] * np.asarray(freqs, np.float64)[None, :]
    c, s = np.cos(a)[:, None, :], np.sin(a)[:, None, :] * (-1.0 if inverse else 1.0)
    one, two = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    p, q = np.asarray(x, np.float64)[..., one], np.asarray(x, np.float64)[..., two]
    with np.errstate(invalid="ignore"):
        out[..., one], out[..., two] = magnitude * (p * c - q * s), magnitude * (q * c + p * s)
    mass[..., one] = mass[..., two] = magnitude * (np.abs(p) + np.abs(q))
    return out, mass


def _code_values():
    i = np.arange(128)
    e, m = i >> 3, i & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v[127] = np.nan
    return np.concatenate([v, -v])


CODES = _code_values()


def encode(x):
    """The e4m3 code nearest to each number of magnitude 448 or less, ties to the even code; 0x7F for NaN and infinities."""
    x = np.asarray(x, np.float64)
    m = np.where(np.isfinite(x), np.abs(x), 0.0)
    up = np.clip(np.searchsorted(CODES[:127], m), 0, 126)
    down = np.maximum(up - 1, 0)
    over, under = CODES[up] - m, m - CODES[down]
    code = np.where((under < over) | ((under == over) & (down % 2 == 0)), down, up)
    code = np.where(np.isfinite(x), code | np.where(np.signbit(x), 128, 0), 127)
    return code.astype(np.uint8)


def block_exp(x):
    """Exponent byte of a block by its numbers: the smallest e >= 1 with |x| <= 448 * 2^(e - 127)."""
    m = np.abs(x[np.isfinite(x)])
    top, e = (m.max() if m.size else 0.0), 1
    while e < 254 and top > 448.0 * 2.0 ** (e - 127):
        e += 1
    return e


def empty_cache(pages, kv_heads, page, dim, fill=0, exp=0):
    return {"k": np.full((pages, kv_heads, page, dim), fill, np.uint8),
            "v": np.full((pages, kv_heads, page // 16, dim, 16), fill, np.uint8),
            "k_exps": np.full((pages, kv_heads), exp, np.uint8), "v_exps": np.full((pages, kv_heads), exp, np.uint8)}


def _rows(cache, name):
    """The codes as [pages, kv_heads, page, dim], a copy of v's."""
    if name == "k":
        return cache["k"]
    pages, heads, page, dim = cache["k"].shape
    return cache["v"].transpose(0, 1, 2, 4, 3).reshape(pages, heads, page, dim)


def append(k, v, cu, lens, table, cache, freqs=None, positions=None, interleaved=False, magnitude=1.0):
    """What the cache holds afterwards (a new dict).  k, v [total, kv_heads, dim] in fp64."""
    cache = {n: t.copy() for n, t in cache.items()}
    pages, heads, page, dim = cache["k"].shape
    total, cap = k.shape[0], table.shape[1] * page
    edges = [min(max(int(c), 0), total) for c in cu]
    for s in range(len(lens)):
        first, last = edges[s], edges[s + 1]
        count, length = max(last - first, 0), max(int(lens[s]), 0)
        places = np.arange(length - count, length)
        new = {"k": k[first:last], "v": v[first:last]}
        if freqs is not None and count:
            at = places if positions is None else np.asarray(positions)[first:last]
            turned = rope(k[first:last], at, freqs, interleaved, False, magnitude)[0]
            new["k"] = np.where(np.abs(turned) >= 2.0 ** 128, np.inf, turned)   # (beyond what a key may be: infinite)
        for p in sorted({int(t) // page for t in places if 0 <= t < cap}):
            here = [i for i, t in enumerate(places) if t >= 0 and t // page == p]
            at, of = int(table[s, p]), int(places[here[0]]) % page
            if not 0 <= at < pages:
                continue
            for name in ("k", "v"):
                rows = _rows(cache, name)[at].copy()
                for h in range(heads):
                    x = new[name][here, h]
                    e, old = block_exp(x), int(cache[name + "_exps"][at, h])
                    if of > 0:
                        e = max(e, old)
                        if e != old:
                            rows[h, :of] = encode(CODES[rows[h, :of]] * 2.0 ** (old - e))
                    rows[h, of:of + len(here)] = encode(x * 2.0 ** (127 - e))
                    cache[name + "_exps"][at, h] = e
                if name == "k":
                    cache["k"][at] = rows
                else:
                    cache["v"][at] = rows.reshape(heads, page // 16, 16, dim).transpose(0, 1, 3, 2)
    return cache


def tokens_of(cache, name, row, n):
    """The numbers of a sequence's first n tokens, [n, kv_heads, dim], and which of them count."""
    pages, heads, page, dim = cache["k"].shape
    codes, exps = _rows(cache, name), cache[name + "_exps"].astype(np.float64)
    out, there = np.zeros((n, heads, dim)), np.zeros(n, bool)
    for i in range(n):
        at = int(row[i // page])
        if 0 <= at < pages:
            out[i], there[i] = CODES[codes[at, :, i % page]] * 2.0 ** (exps[at, :, None] - 127), True
    return out, there


def attn_paged(q, cache, table, lens, scale=None):
    """q [batch, heads, dim]: the output and its error's measure, sum of p |v| / sum of p."""
    batch, heads, dim = q.shape
    kv = cache["k"].shape[1]
    scale = dim ** -0.5 if scale is None else scale
    out, mass = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(batch):
        n = min(max(int(lens[b]), 0), table.shape[1] * cache["k"].shape[2])
        k, there = tokens_of(cache, "k", table[b], n)
        v, _ = tokens_of(cache, "v", table[b], n)
        for h in range(heads):
            g = h // (heads // kv)
            out[b, h], mass[b, h] = _attend(q[b, h], k[there, g], v[there, g], scale)
    return out, mass
