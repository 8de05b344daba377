"""Pins of the fp64 statements of rotary positions and the paged cache: closed forms and brute force."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import paged as OP
from oracle import serving as OS


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_is_a_product_of_complex_numbers(interleaved):
    rng = np.random.default_rng(0)
    x, at, freqs = rng.standard_normal((5, 3, 24)), [0, 1, -7, 100, 1 << 20], 10000.0 ** (-np.arange(8) / 8)
    out, mass = OP.rope(x, at, freqs, interleaved, magnitude=1.5)
    for t in range(5):
        for h in range(3):
            for i in range(8):
                a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + 8)
                z = complex(x[t, h, a], x[t, h, b]) * np.exp(1j * at[t] * freqs[i]) * 1.5
                assert out[t, h, a] == pytest.approx(z.real, abs=1e-9) and out[t, h, b] == pytest.approx(z.imag, abs=1e-9)
                assert mass[t, h, a] == mass[t, h, b] == 1.5 * (abs(x[t, h, a]) + abs(x[t, h, b]))
    assert (out[..., 16:] == x[..., 16:]).all()
    assert np.allclose(OP.rope(out, at, freqs, interleaved, inverse=True, magnitude=1 / 1.5)[0], x)


def test_rope_scores_depend_on_the_distance_alone():
    rng = np.random.default_rng(1)
    q, k, freqs = rng.standard_normal((1, 1, 16)), rng.standard_normal((1, 1, 16)), 0.3 ** np.arange(8)
    score = lambda i, j: (OP.rope(q, [i], freqs)[0] * OP.rope(k, [j], freqs)[0]).sum()
    assert score(5, 2) == pytest.approx(score(1003, 1000))


def test_rope_inverse_is_the_transpose():
    """Against differences: d sum(w rope(x)) / dx is rope's inverse of w."""
    rng = np.random.default_rng(2)
    x, w, at, freqs = rng.standard_normal((2, 1, 16)), rng.standard_normal((2, 1, 16)), [3, 11], 0.5 ** np.arange(6)
    f = lambda x: (w * OP.rope(x, at, freqs, True, magnitude=1.25)[0]).sum()
    g = OP.rope(w, at, freqs, True, inverse=True, magnitude=1.25)[0]
    for i in np.ndindex(x.shape):
        d = np.zeros_like(x)
        d[i] = 1e-4
        assert (f(x + d) - f(x - d)) / 2e-4 == pytest.approx(g[i], abs=1e-8)


def test_codes_are_those_of_the_format():
    for i in range(127):
        e, m = i >> 3, i & 7
        assert Fraction(OP.CODES[i]) == (Fraction(m, 512) if e == 0 else (1 + Fraction(m, 8)) * Fraction(2) ** (e - 7))
        assert OP.CODES[128 + i] == -OP.CODES[i]
    assert OP.CODES[126] == 448 and np.isnan(OP.CODES[[127, 255]]).all()


def test_encode_by_brute_force():
    rng = np.random.default_rng(3)
    x = np.concatenate([OP.CODES[:127], rng.uniform(-448, 448, 100), rng.standard_normal(100) * 0.02,
                        (OP.CODES[:126] + OP.CODES[1:127]) / 2, -(OP.CODES[:126] + OP.CODES[1:127]) / 2])
    finite = [*range(127), *range(128, 255)]
    codes = [Fraction(OP.CODES[i]) for i in finite]
    for v, c in zip(x, OP.encode(x)):
        d = [abs(Fraction(v) - y) for y in codes]
        least = min(d)
        best = [i for i, e in zip(finite, d) if e == least]
        assert c in best and (len({OP.CODES[b] for b in best}) == 1 or c % 2 == 0)
    assert (OP.encode([np.nan, np.inf, -np.inf]) == 127).all()


def test_block_exponent_is_the_smallest_that_fits():
    for top in (448.0, 448.0000001, 1.75, 1.7500001, 1.0, 3.5e-3, 0.0, 2.0 ** -130, 3e38):
        e = OP.block_exp(np.array([[0.5 * top, -top], [np.nan, np.inf]]))
        assert top <= 448 * 2.0 ** (e - 127) and (e == 1 or top > 448 * 2.0 ** (e - 128))


@pytest.mark.parametrize("page", [16, 32])
def test_append_token_by_token_is_append_at_once_where_blocks_do_not_grow(page):
    """The largest numbers first: the exponents that the first token sets hold, and so does every code."""
    rng = np.random.default_rng(4)
    n, heads, dim = 2 * page + 3, 2, 64
    x = rng.uniform(-1, 1, (n, heads, dim))
    x[::page] *= 1.9 / np.abs(x[::page]).max((1, 2), keepdims=True)
    x[::page, :, 0] = 1.9
    table, cu = np.array([[2, 0, 1]]), [0, n]
    whole = OP.append(x, 0.5 * x, cu, [n], table, OP.empty_cache(3, heads, page, dim))
    step = OP.empty_cache(3, heads, page, dim)
    for i in range(n):
        step = OP.append(x[i:i + 1], 0.5 * x[i:i + 1], [0, 1], [i + 1], table, step)
    assert all((whole[name] == step[name]).all() for name in whole)
    got, there = OP.tokens_of(whole, "k", table[0], n)
    assert there.all() and (np.abs(got - x) <= 2.0 ** -4 * np.abs(x) + 1.9 * 2.0 ** -17).all()


def test_append_that_grows_a_block_moves_the_codes():
    x = np.zeros((3, 1, 64))
    x[0, 0, :4], x[1, 0, :2], x[2, 0, 0] = [1.0, -0.5, 2.0 ** -6, 2.0 ** -9], [3.0, 100.0], 7.0
    cache = OP.empty_cache(1, 1, 16, 64, fill=0x33)
    table = np.array([[0]])
    for i in range(3):
        cache = OP.append(x[i:i + 1], x[i:i + 1], [0, 1], [i + 1], table, cache)
    assert (cache["k_exps"] == 127 - 2).all()              # 100 <= 448 / 4
    assert (cache["k"][0, 0, 3:] == 0x33).all() and (cache["v"][0, 0, 0, :, 3:] == 0x33).all()
    got, _ = OP.tokens_of(cache, "v", [0], 3)
    x[1, 0, 1] = 96                                        # (half-way between 96 and 104)
    assert (got[:, 0, :2] == x[:, 0, :2]).all() and got[0, 0, 2] == 2.0 ** -6
    assert got[0, 0, 3] == 2.0 ** -9                       # (0x01 of the smallest exponent on the way: 2^-9 / 2^-2 is 2^-7)


def test_append_leaves_what_it_does_not_write():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((6, 1, 64))
    before = OP.empty_cache(3, 1, 16, 64, fill=7, exp=120)
    after = OP.append(x, x, [0, 2, 2, 6], [2, 0, 18], np.array([[9, 9], [1, 1], [2, -1]]), before)
    assert (after["k"][:2] == 7).all() and (after["k_exps"][:2] == 120).all()   # page 9 does not exist, nothing is page 1's
    assert (after["k"][2, 0, :14] == OP.encode(OP.CODES[7] * 2.0 ** (120.0 - after["k_exps"][2, 0]))).all()
    got, there = OP.tokens_of(after, "k", [2, -1], 18)
    assert there[:16].all() and not there[16:].any() and np.abs(got[14:16] - x[2:4]).max() < 0.2


def test_attention_over_pages_is_attention_over_a_row_of_tokens():
    rng = np.random.default_rng(6)
    lens, table, heads, kv, dim, page = [37, 0, 16], np.array([[4, 0, 2], [1, 1, 1], [3, 7, 7]]), 4, 2, 64, 16
    cache = OP.empty_cache(5, kv, page, dim)
    for name in ("k", "v"):
        cache[name] = OP.encode(rng.uniform(-3, 3, cache[name].shape))
        cache[name + "_exps"] = rng.integers(125, 129, cache[name + "_exps"].shape).astype(np.uint8)
    q = rng.standard_normal((3, heads, dim))
    out, mass = OP.attn_paged(q, cache, table, lens)
    own = {}
    for name in ("k", "v"):
        own[name] = np.zeros((3, 48, kv, dim))
        for b, n in enumerate(lens):
            for i in range(n):
                for d in range(dim):
                    p, t = table[b, i // page], i % page
                    c = cache["k"][p, :, t, d] if name == "k" else cache["v"][p, :, t // 16, d, t % 16]
                    own[name][b, i, :, d] = OP.CODES[c] * 2.0 ** (cache[name + "_exps"][p].astype(float) - 127)
    none = np.zeros((0, kv, dim))
    want, want_mass = OS.attn_prefix(q, none, none, own["k"], own["v"], lens)
    assert np.allclose(out, want) and np.allclose(mass, want_mass) and (out[1] == 0).all()


def test_keys_that_turn_past_the_largest_count_as_infinite():
    """2^128 and beyond, by the turn or by the magnitude: NaN in the cache, and not counted for the block's exponent."""
    big, k = 1.5 * 2.0 ** 127, np.zeros((3, 1, 16))
    k[0, 0, 0], k[0, 0, 8] = big, big                      # a turn by 1: sum and difference, 1.38 and 0.30 times as much
    k[1, 0, 1] = 2.0 ** 127                                # twice that is 2^128 itself
    k[2, 0, 2] = 2.0 ** 127 * (1 - 2.0 ** -8)              # and this stays below
    freqs, table = np.array([1.0, 0, 0, 0, 0, 0, 0, 0]), np.array([[0]])
    got = OP.append(k, k, [0, 3], [3], table, OP.empty_cache(1, 1, 16, 16), freqs, [1, 0, 0], magnitude=2.0)
    x = OP.CODES[got["k"][0, 0]] * 2.0 ** (got["k_exps"][0, 0] - 127.0)
    a = 2 * big * (np.sin(1.0) + np.cos(1.0))
    assert a >= 2.0 ** 128 and 2 * big * (np.sin(1.0) - np.cos(1.0)) < 2.0 ** 128
    assert np.isnan(x[0, 8]) and np.isfinite(x[0, 0]) and np.isnan(x[1, 1]) and np.isfinite(x[2]).all() and x[2, 2] == 2.0 ** 128
    assert got["k_exps"][0, 0] == OP.block_exp(np.array([2.0 ** 128 * (1 - 2.0 ** -8)]))
