"""Pins of the fp64 statements of the serving operators: closed forms and brute force."""
import math

import numpy as np
import pytest

from oracle import serving as OS


def test_prompt_attention_of_equal_keys_is_the_running_mean():
    rng = np.random.default_rng(0)
    v = rng.standard_normal((9, 1, 4))
    out, mass = OS.attn_prompt(rng.standard_normal((9, 2, 4)), np.zeros((9, 1, 4)), v, [1, 4, 4, 8])
    for a, b in ((1, 4), (4, 8)):
        for i in range(a, b):
            for h in range(2):
                assert np.allclose(out[i, h], v[a:i + 1, 0].mean(0))
                assert np.allclose(mass[i, h], np.abs(v[a:i + 1, 0]).mean(0))
    assert np.isnan(out[[0, 8]]).all()


def test_prompt_attention_by_brute_force():
    rng = np.random.default_rng(1)
    q, k, v = (rng.standard_normal((5, h, 3)) for h in (4, 2, 2))
    out, _ = OS.attn_prompt(q, k, v, [0, 5], scale=0.7)
    for i in range(5):
        for h in range(4):
            w = [math.exp(0.7 * sum(q[i, h, d] * k[j, h // 2, d] for d in range(3))) for j in range(i + 1)]
            for d in range(3):
                want = sum(w[j] * v[j, h // 2, d] for j in range(i + 1)) / sum(w)
                assert out[i, h, d] == pytest.approx(want, rel=1e-12)


def test_prefix_attention_is_the_last_row_of_the_whole_prompt():
    rng = np.random.default_rng(2)
    p, cap, lens = 6, 5, [0, 3, 9, -2]
    K, V = rng.standard_normal((2, p, 2, 8))
    Ko, Vo = rng.standard_normal((2, 4, cap, 2, 8))
    q = rng.standard_normal((4, 6, 8))
    out, _ = OS.attn_prefix(q, K, V, Ko, Vo, lens)
    for b, n in enumerate([0, 3, 5, 0]):
        k, v = np.concatenate([K, Ko[b, :n]]), np.concatenate([V, Vo[b, :n]])
        rows = np.zeros((p + n, 6, 8))
        rows[-1] = q[b]
        whole, _ = OS.attn_prompt(rows, k, v, [0, p + n])
        assert np.allclose(out[b], whole[-1], rtol=1e-12)
    none, mass = OS.attn_prefix(q, K[:0], V[:0], Ko, Vo, lens)
    assert (none[[0, 3]] == 0).all() and (mass[[0, 3]] == 0).all()


def test_w4_codes_bit_by_bit_and_product_of_ones():
    rng = np.random.default_rng(3)
    n, k = 37, 264
    codes = rng.integers(0, 16, (n, k))
    words = np.zeros((3, 3, 64, 4), np.int64)
    for r in range(n):
        for c in range(k):
            i, q, e = c % 128 // 32, c % 32 // 8, c % 8
            words[r // 16, c // 128, 16 * q + r % 16, i] |= int(codes[r, c]) << (4 * (e // 2) + 16 * (e % 2))
    words = np.where(words >= 1 << 31, words - (1 << 32), words).astype(np.int32)
    assert (OS.w4_codes(words, n, k) == codes).all()
    y, mass = OS.gemv_w4(np.ones((2, k)), codes, np.ones((n, 3)), np.full((n, 3), 2), 128)
    assert (y == (codes - 2).sum(1)).all() and (mass == (codes + 258).sum(1)).all()
    y, _ = OS.gemv_w4(np.ones((1, k)), codes, np.full((n, 9), 0.5), None, 32)
    assert (y == ((codes - 8) * 0.5).sum(1)).all()
