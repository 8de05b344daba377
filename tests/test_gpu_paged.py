"""GPU parity of rotary positions and the paged 8-bit cache against their fp64 statements, in every launch form, at
the sizes and masks where they can go wrong.

Tolerances, all of them from the arithmetic.  bf16 rounds by at most 2^-8 of a value, fp32 by 2^-24.
  rope: sine, cosine and two operations on them are rounded to fp32, then the output once:
    |d| <= 2^-8 |want| + 4 x 2^-24 x 1.01 M, with M = magnitude (|x1| + |x2|).
  append: keys are turned in fp64 and rounded once, so codes and exponents are the oracle's.  (Both sides' fp64 differs
    by some 2^-48; that a number of the inputs here lies as near to a border of two codes has odds of 2^-30.)
  attention: as for prompts, |d| <= 2^-8 |want| + (2^-8 + 2^-12) M, with M = sum p |v| / sum p: the output is rounded once,
    each p once before the second product; codes enter the products exactly.  2^-12 covers fp32 while scores stay
    below 20 and tokens below 4096 a sequence.
"""
import numpy as np
import pytest

import tally_inputs as TI
from oracle import bf16 as obf16
from oracle import paged as OP
from oracle import serving as OS

pytestmark = pytest.mark.gpu
SENTINEL = 0x7ABC                                          # a bf16 that no output is
FORMS = ["hi", "be", "sliced", "ptb"]


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2410_07381_amd.binding as B
    assert torch.cuda.is_available()
    hi, be = torch.cuda.Stream(), torch.cuda.Stream()
    ctx = B.Context(hi, be)
    yield B, ctx, torch
    ctx.close()


def _bits(rng, shape, scale=1.0):
    return TI.to_bf16_bits((rng.standard_normal(shape) * scale).astype(np.float32))


def _dev(torch, bits):
    a = np.ascontiguousarray(bits)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()


def _host(t):
    a = t.cpu().numpy()
    return a.view(np.uint16) if a.dtype == np.int16 else a


def _run(ctx, torch, kernel, form):
    """The whole kernel in one of its forms."""
    torch.cuda.synchronize()
    if form in ("hi", "be"):
        ctx.launch_native(kernel, hi=form == "hi")
    elif form == "sliced":
        job = ctx.launch_sliced(kernel, max(kernel.total_blocks // 3, 1))
        while job.wait() != 3:
            job.resume()
        job.free()
    else:
        total = kernel.total_blocks
        job = ctx.launch_ptb(kernel, min(ctx.max_workers(kernel), max(total // 2, 1)), coverage=True, stop_at=total // 2)
        job.wait()
        assert job.progress()[0] == total // 2 or job.progress()[2] == 3
        job.resume()
        assert job.wait() == 3
        assert (job.coverage()["count"] == 1).all()
        job.free()
    torch.cuda.synchronize()


# ---------------------------------------------------------------- rotary positions
def _rope_ok(got_bits, want, mass):
    got = obf16.decode(got_bits)
    bound = 2.0 ** -8 * np.abs(want) + 4.04 * 2.0 ** -24 * mass
    err = np.abs(got - want)
    assert (err <= bound).all(), f"{(err > bound).sum()} of {err.size} off; worst {(err / np.maximum(bound, 1e-30)).max():.2f} bounds"


ROPE = [(1, 1, 64, 64), (1, 24, 64, 64), (3, 5, 128, 32), (7, 1, 16, 16), (33, 3, 80, 48), (5, 2, 96, 96), (17, 40, 128, 128), (2, 2, 512, 512),
        (1030, 1, 128, 64), (4111, 2, 64, 32), (70001, 1, 16, 16)]


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("total,heads,dim,rot", ROPE)
def test_rope(env, total, heads, dim, rot, form):
    B, ctx, torch = env
    rng = np.random.default_rng(total + dim)
    interleaved, inverse = bool(total % 2), form in ("be", "ptb")
    # heads in front of others, rows with something between them
    x = _bits(rng, (total, heads + 3, dim))
    at = rng.integers(-100, 1 << 20, total).astype(np.int32)
    at[0] = 0 if total == 1 else (1 << 31) - 1
    freqs = (10000.0 ** (-np.arange(rot // 2) / (rot // 2))).astype(np.float32)
    tx, tf, ta = _dev(torch, x), _dev(torch, freqs), _dev(torch, at)
    out = torch.full((total, heads + 1, dim), SENTINEL, dtype=torch.int16, device="cuda")
    _run(ctx, torch, B.rope_bf16(tx[:, :heads], out[:, :heads], tf, ta, interleaved, inverse, magnitude=1.25), form)
    want, mass = OP.rope(obf16.decode(x[:, :heads]), at, freqs, interleaved, inverse, 1.25)
    _rope_ok(_host(out)[:, :heads], want, mass)
    assert (_host(out)[:, heads:] == SENTINEL).all() and (_host(tx) == x).all()
    assert (_host(out)[:, :heads, rot:] == x[:, :heads, rot:]).all()   # copied, not computed
    _run(ctx, torch, B.rope_bf16(tx[:, :heads], tx[:, :heads], tf, ta, interleaved, inverse, magnitude=1.25), form)   # in place
    assert (_host(tx)[:, :heads] == _host(out)[:, :heads]).all() and (_host(tx)[:, heads:] == x[:, heads:]).all()


def test_rope_far_positions_and_numbers_that_are_none(env):
    B, ctx, torch = env
    rng = np.random.default_rng(1)
    x = _bits(rng, (6, 2, 64))
    x[1, 0, 3], x[2, 1, 40], x[3, 0, 63] = 0x7F80, 0x7FC0, 0xFF80
    at = np.array([(1 << 31) - 1, -(1 << 31), 1 << 29, 12345677, 0, -1], np.int32)
    freqs = np.array([1.0, 0.9999, 1e-3, 0.0, 0.37, 1e-6, 0.5, 0.123] * 4, np.float32)
    tx, out = _dev(torch, x), torch.zeros((6, 2, 64), dtype=torch.int16, device="cuda")
    _run(ctx, torch, B.rope_bf16(tx, out, _dev(torch, freqs), _dev(torch, at)), "hi")
    with np.errstate(invalid="ignore"):
        want, mass = OP.rope(obf16.decode(x), at, freqs)
    fine = np.isfinite(mass)
    got = obf16.decode(_host(out))
    assert not np.isfinite(got[~fine]).any()
    # angles near 2^31 are off by 2^-23 in the product, as the oracle's are
    err = np.abs(got - np.where(fine, want, 0))[fine]
    assert (err <= 2.0 ** -8 * np.abs(want[fine]) + (4.04 * 2.0 ** -24 + 2.0 ** -22) * mass[fine]).all()


def test_rope_inverse_is_the_gradient(env):
    """Against differences of the operator itself: it is linear, so sum w (rope(x + d) - rope(x - d)) is 2 sum rope'(w) d."""
    B, ctx, torch = env
    rng = np.random.default_rng(2)
    shape, freqs = (9, 3, 64), (0.7 ** np.arange(24)).astype(np.float32)
    at = rng.integers(0, 5000, 9).astype(np.int32)
    tf, ta = _dev(torch, freqs), _dev(torch, at)

    def call(bits, **how):
        out = torch.zeros(shape, dtype=torch.int16, device="cuda")
        _run(ctx, torch, B.rope_bf16(_dev(torch, bits), out, tf, ta, **how), "hi")
        return obf16.decode(_host(out))
    w = _bits(rng, shape)
    g = call(w, inverse=True, magnitude=1.5)
    _, mass = OP.rope(obf16.decode(w), at, freqs, magnitude=1.5)
    for i in range(8):
        d = np.zeros(shape)
        d[tuple(rng.integers(0, n) for n in shape)] = 1.0
        plus, minus = (call(TI.to_bf16_bits((s * d).astype(np.float32)), magnitude=1.5) for s in (1.0, -1.0))
        got, want = (obf16.decode(w) * (plus - minus)).sum() / 2, (g * d).sum()
        # the column's two numbers and the gradient's are rounded once each
        assert abs(got - want) <= 2.0 ** -7 * (mass * d).sum() * 1.01


# ---------------------------------------------------------------- appending
def _cache(rng, pages, kv, page, dim, lo=118, hi=123):
    c = {"k": rng.integers(0, 256, (pages, kv, page, dim)).astype(np.uint8), "v": rng.integers(0, 256, (pages, kv, page // 16, dim, 16)).astype(np.uint8)}
    for n in ("k", "v"):
        c[n][(c[n] & 127) == 127] = 0x70
        c[n + "_exps"] = rng.integers(lo, hi + 1, (pages, kv)).astype(np.uint8)
    return c


def _paged(B, torch, cache):
    return B.PagedCache(*(_dev(torch, cache[n]) for n in ("k", "v", "k_exps", "v_exps")))


def _same(got, want, name=""):
    for n, t in zip(("k", "v", "k_exps", "v_exps"), got):
        g, w = _host(t), want[n]
        if n in ("k", "v"):                                # (zeros of either sign, any NaN)
            g, w = np.nan_to_num(OP.CODES[g], nan=1e9), np.nan_to_num(OP.CODES[w], nan=1e9)
        assert (g == w).all(), f"{name} {n}: {(g != w).sum()} of {g.size} differ, first at {np.argwhere(g != w)[0]}"


def _deal(rng, lens, page, spare=2, more=0):
    """A table of pages in no order, and how many there are."""
    need = [-(-int(n) // page) for n in lens]
    ids = rng.permutation(sum(need) + spare).astype(np.int32)
    table = np.full((len(lens), max(max(need), 1) + more), -1, np.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = ids[at:at + n]
        at += n
    return table, sum(need) + spare


APPEND = [
    # new tokens, tokens held before, kv heads, dim, page, rot
    ([1], [0], 1, 64, 16, 64), ([1], [15], 1, 128, 16, 128), ([1], [16], 2, 128, 32, 0), ([1], [1000], 8, 128, 64, 128), ([2], [15], 3, 64, 16, 32),
    ([16], [0], 5, 128, 16, 64), ([17], [15], 4, 64, 16, 16), ([100], [7], 1, 128, 128, 128), ([300], [65], 2, 64, 128, 64), ([129], [63], 2, 128, 64, 96),
    ([1, 1, 1, 1, 1], [0, 5, 15, 16, 31], 8, 128, 16, 128), ([0, 3, 0, 0, 40, 1], [9, 30, 0, 16, 1, 127], 3, 64, 32, 48),
    ([64, 0, 65, 1], [64, 64, 0, 63], 1, 64, 64, 64), ([5, 200, 31], [0, 100, 33], 7, 128, 32, 128), ([255, 1], [1, 127], 2, 64, 128, 0),
    ([1] * 70, list(range(70)), 1, 64, 16, 64), ([1, 0, 2] * 50, [3] * 150, 2, 64, 16, 32),
    # mostly one token, and one sequence that gets many: its pages are gone through by one wave, or four
    ([1] * 30 + [0] * 260 + [250], [60 + i for i in range(291)], 2, 128, 128, 128), ([1] * 30 + [0] * 260 + [250], [5] * 291, 1, 64, 64, 48),
    ([2] * 20 + [130], [126 - i for i in range(21)], 3, 128, 128, 128), ([3, 1, 60, 1, 0, 2] * 4, [62, 13, 100, 0, 0, 127] * 4, 1, 128, 64, 64),
    ([3, 1, 100, 1, 0, 2] * 4, [62, 13, 100, 0, 0, 127] * 4, 2, 64, 128, 16),
]


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("new,held,kv,dim,page,rot", APPEND)
def test_append(env, new, held, kv, dim, page, rot, form):
    B, ctx, torch = env
    rng = np.random.default_rng(sum(new) + 7 * page + dim)
    cu, behind = np.concatenate([[0], np.cumsum(new)]).astype(np.int32), 3
    total = int(cu[-1]) + behind
    x = _bits(rng, (total, 2 * kv + 1, dim))
    lens = (np.array(new) + held).astype(np.int32)
    table, pages = _deal(rng, lens, page, more=1)
    cache = _cache(rng, pages, kv, page, dim)
    freqs = (10000.0 ** (-np.arange(rot // 2) / max(rot // 2, 1))).astype(np.float32) if rot else None
    interleaved = kv % 2 == 0
    positions = rng.integers(0, 1 << 20, total).astype(np.int32) if rot and len(new) % 2 == 0 else None
    tx, t = _dev(torch, x), lambda a: None if a is None else _dev(torch, a)
    paged = _paged(B, torch, cache)
    kern = B.kv_append_fp8(tx[:, :kv], tx[:, kv:2 * kv], t(cu), t(lens), t(table), paged, t(freqs), t(positions), interleaved,
                           magnitude=1.2 if rot else None)
    k, v = obf16.decode(x[:, :kv]), obf16.decode(x[:, kv:2 * kv])
    want = OP.append(k, v, cu, lens, table, cache, freqs, positions, interleaved, float(np.float32(1.2)))   # (as the call takes it)
    _run(ctx, torch, kern, form)
    _same(paged, want, form)
    _run(ctx, torch, kern, form)                           # again: what was left the first time
    _same(paged, want, "again")


@pytest.mark.parametrize("new,held,kv,dim,page,rot,form", [
    ([17000], [0], 4, 128, 64, 128, "hi"), ([33000], [5], 8, 128, 32, 64, "ptb"), ([23000], [100], 3, 128, 128, 128, "sliced"),
    ([9000, 1, 13000], [3, 500, 17], 7, 64, 16, 64, "ptb"), ([40000], [0], 5, 64, 128, 0, "hi")])
def test_append_with_several_heads_a_wave(env, new, held, kv, dim, page, rot, form):
    """Calls so large that a wave goes through two heads, or four, one after the other; numbers of heads that they do not divide."""
    test_append(env, new, held, kv, dim, page, rot, form)


@pytest.mark.parametrize("form", FORMS)
def test_thousands_of_sequences(env, form):
    """More of them than two rounds of 63 find: appended to, few tokens each and most of them none, and attended to."""
    B, ctx, torch = env
    rng = np.random.default_rng(21)
    n, page, dim = 5000, 16, 64
    new, held = (rng.random(n) < 0.3).astype(int), rng.integers(0, 40, n)
    new[[7, 4990]] = 45
    lens = (new + held).astype(np.int32)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    table, pages = _deal(rng, lens, page)
    cache = _cache(rng, pages, 1, page, dim)
    x, q = _bits(rng, (int(cu[-1]), 2, dim)), _bits(rng, (n, 1, dim), 0.25)
    paged, tx, tt, tl = _paged(B, torch, cache), _dev(torch, x), _dev(torch, table), _dev(torch, lens)
    _run(ctx, torch, B.kv_append_fp8(tx[:, :1], tx[:, 1:], _dev(torch, cu), tl, tt, paged), form)
    cache = OP.append(obf16.decode(x[:, :1]), obf16.decode(x[:, 1:]), cu, lens, table, cache)
    _same(paged, cache)
    if form in ("hi", "be"):
        scratch = torch.zeros(max(B.attn_paged_scratch_bytes(n, 1, 1, dim, page, table.shape[1]), 1), dtype=torch.uint8, device="cuda")
        out = torch.zeros((n, 1, dim), dtype=torch.int16, device="cuda")
        _run(ctx, torch, B.attn_paged_fp8(_dev(torch, q), paged, tt, tl, out, scratch, scale=0.02), form)
        _attn_ok(_host(out), *OP.attn_paged(obf16.decode(q), cache, table, lens, 0.02))


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("dim", [64, 128])
def test_append_numbers_of_every_size(env, dim, page):
    """Zeros, subnormals, the largest, NaN and infinities; blocks whose largest is a border of two exponents, or next to one."""
    B, ctx, torch = env
    rng = np.random.default_rng(3)
    n = 8 * page
    x = _bits(rng, (n, 2, dim))
    tops = [0.0, 2.0 ** -133, 2.0 ** -126, 1.75, 1.7578125, 448.0, 450.0, 3.3e38]
    for i, top in enumerate(tops):                         # one page each
        rows = obf16.decode(x[i * page:(i + 1) * page])
        rows = np.clip(rows / 4, -1, 1) * top * 0.99
        rows[3, :, 5] = top
        x[i * page:(i + 1) * page] = TI.to_bf16_bits(rows.astype(np.float32))
    x[page + 1, 0, 7], x[2 * page + 2, 1, 9], x[5, 0, 0] = 0x7F80, 0x7FC0, 0xFF80
    x[6 * page:6 * page + 2, :, :] = 0x8000                # zeros of the other sign
    cu, lens = np.array([0, n], np.int32), np.array([n], np.int32)
    table, pages = _deal(rng, lens, page)
    cache = _cache(rng, pages, 1, page, dim)
    paged = _paged(B, torch, cache)
    _run(ctx, torch, B.kv_append_fp8(_dev(torch, x[:, :1]), _dev(torch, x[:, 1:]), _dev(torch, cu), _dev(torch, lens), _dev(torch, table), paged), "hi")
    with np.errstate(invalid="ignore", over="ignore"):
        want = OP.append(obf16.decode(x[:, :1]), obf16.decode(x[:, 1:]), cu, lens, table, cache)
    _same(paged, want)
    one = B.PagedCache(*(t.clone() for t in paged)).values()[0].cpu().numpy()
    assert (one[table[0, 5], 0, 3, 5], one[table[0, 3], 0, 3, 5]) == (448.0, 1.75)


def test_append_one_by_one_with_blocks_that_grow(env):
    """Tokens of rising size, one call each: exponents and codes as the oracle's after every one."""
    B, ctx, torch = env
    rng = np.random.default_rng(4)
    n, kv, dim, page = 40, 2, 128, 32
    x = TI.to_bf16_bits((rng.standard_normal((n, 2 * kv, dim)) * 1.4 ** np.arange(n)[:, None, None]).astype(np.float32))
    table, pages = _deal(rng, [n], page)
    cache = _cache(rng, pages, kv, page, dim, 1, 254)      # (what a page held before it was this sequence's does not count)
    paged, tx, tt = _paged(B, torch, cache), _dev(torch, x), _dev(torch, table)
    freqs = (0.5 ** np.arange(64)).astype(np.float32)
    tf, cu = _dev(torch, freqs), _dev(torch, np.array([0, 1], np.int32))
    for i in range(n):
        lens = np.array([i + 1], np.int32)
        _run(ctx, torch, B.kv_append_fp8(tx[i:i + 1, :kv], tx[i:i + 1, kv:], cu, _dev(torch, lens), tt, paged, tf), "hi")
        cache = OP.append(obf16.decode(x[i:i + 1, :kv]), obf16.decode(x[i:i + 1, kv:]), [0, 1], lens, table, cache, freqs)
        _same(paged, cache, f"token {i}")


@pytest.mark.parametrize("page", [16, 64, 128])
def test_append_as_workers_of_its_own_variant(env, page):
    """As many workers as are resident of the kernel that the sizes take, not of the largest; no more are accepted; the candidates
    go up to them."""
    B, ctx, torch = env
    rng = np.random.default_rng(23)
    n, kv, dim = 6000, 8, 128
    table, pages = _deal(rng, [n], page)
    cache, x = OP.empty_cache(pages, kv, page, dim), _bits(rng, (n, 2 * kv, dim))
    paged, tx = _paged(B, torch, cache), _dev(torch, x)
    cu, lens = _dev(torch, np.array([0, n], np.int32)), _dev(torch, np.array([n], np.int32))
    kern = B.kv_append_fp8(tx[:, :kv], tx[:, kv:], cu, lens, _dev(torch, table), paged)
    most, units = ctx.max_workers(kern), B.device_info()["num_cus"]
    assert most == units if page == 128 else most >= (3 if page == 16 else 1) * units
    configs = [c for c in ctx.candidate_configs(kern) if c[0] == B.CFG_PTB]
    assert max(c[1] for c in configs) == min(most, kern.total_blocks)
    with pytest.raises(B.TallyError) as e:
        ctx.launch_ptb(kern, most + 1)
    assert e.value.status == B.ERR_INVALID_ARG
    torch.cuda.synchronize()
    job = ctx.launch_ptb(kern, min(most, kern.total_blocks), coverage=True)
    assert job.wait() == 3 and (job.coverage()["count"] == 1).all()
    job.free()
    torch.cuda.synchronize()
    _same(paged, OP.append(obf16.decode(x[:, :kv]), obf16.decode(x[:, kv:]), [0, n], [n], table, cache))


def test_append_skips_what_has_no_place(env):
    """Pages that do not exist, places before the first and behind the last page, sequences that are empty or out of order."""
    B, ctx, torch = env
    rng = np.random.default_rng(5)
    kv, dim, page, total = 2, 64, 16, 120
    cu = np.array([-5, 20, 20, 60, 50, 90, 500], np.int32)   # (the fourth ends before it begins)
    lens = np.array([10, 0, 60, 5, 1 << 30, -7], np.int32)   # (the first holds fewer than it gets, the fifth ends far behind its pages)
    table = np.array([[3, 1, 0, 0], [0, 0, 0, 0], [2, -1, 7, 4], [5, 5, 5, 5], [6, 6, 6, 6], [6, 6, 6, 6]], np.int32)
    cache = _cache(rng, 7, kv, page, dim)
    x = _bits(rng, (total, 2 * kv, dim))
    paged, tx = _paged(B, torch, cache), _dev(torch, x)
    guard = torch.full((1 << 16,), 77, dtype=torch.uint8, device="cuda")
    kern = B.kv_append_fp8(tx[:, :kv], tx[:, kv:], _dev(torch, cu), _dev(torch, lens), _dev(torch, table), paged)
    _run(ctx, torch, kern, "hi")
    want = OP.append(obf16.decode(x[:, :kv]), obf16.decode(x[:, kv:]), cu, lens, table, cache)
    _same(paged, want)
    assert (want["k"][1] == cache["k"][1]).all() and (want["k"][3] != cache["k"][3]).any() and (guard == 77).all()


# ---------------------------------------------------------------- attention
def _attn_ok(got_bits, want, mass):
    got = obf16.decode(got_bits)
    bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -12) * mass
    assert np.isfinite(got).all()
    err = np.abs(got - want)
    assert (err <= bound).all(), f"{(err > bound).sum()} of {err.size} off; worst {(err / np.maximum(bound, 1e-30)).max():.2f} bounds"


def _filled(rng, pages, kv, page, dim):
    """Codes of normal numbers, exponents that differ from block to block, keys so that scores stay small."""
    c = OP.empty_cache(pages, kv, page, dim)
    for n in ("k", "v"):
        c[n] = OP.encode(np.clip(rng.standard_normal(c[n].shape) * 100, -448, 448))
        c[n + "_exps"] = rng.integers(118, 122, c[n + "_exps"].shape).astype(np.uint8)
    return c


def _attend(B, ctx, torch, q, cache, table, lens, form="hi", scale=None, dirty=True):
    batch, heads, dim = q.shape
    paged, tt, tl = _paged(B, torch, cache), _dev(torch, table), _dev(torch, np.asarray(lens, np.int32))
    pages, kv, page, _ = cache["k"].shape
    size = B.attn_paged_scratch_bytes(batch, heads, kv, dim, page, table.shape[1])
    scratch = torch.full((max(size, 1),), 0xFF if dirty else 0, dtype=torch.uint8, device="cuda")   # (NaN throughout)
    out = torch.full((batch + 1, heads + 1, dim), SENTINEL, dtype=torch.int16, device="cuda")
    _run(ctx, torch, B.attn_paged_fp8(_dev(torch, q), paged, tt, tl, out[:batch, :heads], scratch, scale), form)
    got = _host(out)
    assert (got[batch] == SENTINEL).all() and (got[:, heads] == SENTINEL).all()
    return got[:batch, :heads]


PAGED = [
    # tokens, heads, kv heads, dim, page, pages of a row beyond what the longest needs
    ([1], 1, 1, 64, 16, 0), ([0], 2, 1, 128, 16, 0), ([1, 0], 2, 2, 128, 32, 1), ([15, 16, 17], 3, 1, 64, 16, 0), ([31, 32, 33], 4, 4, 128, 16, 3),
    ([63, 64, 65, 127, 128, 129], 8, 2, 128, 64, 0), ([255, 256, 257], 7, 1, 64, 128, 0), ([511, 512, 513], 5, 5, 64, 16, 0),
    ([1000, 0, 3, 700], 32, 8, 128, 64, 0), ([3001, 1, 2000], 28, 4, 128, 32, 0), ([2500], 16, 1, 128, 128, 0), ([1500, 100], 17, 1, 64, 32, 0),
    ([900, 33], 40, 1, 128, 16, 0), ([4000], 2, 2, 64, 64, 0), ([40, 300], 12, 12, 64, 16, 400), ([600, 5, 0, 77], 96, 2, 64, 16, 40),
    ([20 * i % 97 for i in range(70)], 2, 1, 64, 16, 0), ([700 + i for i in range(40)], 8, 8, 64, 64, 8), ([1500, 3, 900] * 2, 4, 4, 128, 32, 70000), ([1] * 63 + [0] * 66 + [900], 1, 1, 64, 16, 0), ([130 + i for i in range(65)], 2, 2, 64, 32, 30),
]


@pytest.mark.parametrize("form", ["hi", "be"])
@pytest.mark.parametrize("lens,heads,kv,dim,page,more", PAGED)
def test_attention(env, lens, heads, kv, dim, page, more, form):
    B, ctx, torch = env
    rng = np.random.default_rng(sum(lens) + heads + page)
    table, pages = _deal(rng, lens, page, more=more)
    cache, q = _filled(rng, pages, kv, page, dim), _bits(rng, (len(lens), heads, dim))
    want, mass = OP.attn_paged(obf16.decode(q), cache, table, lens)
    # what lies behind the lengths does not count, whatever it is: entries of the table (-1 here), tokens in the last page
    for b, n in enumerate(lens):
        if n % page:
            at, t = table[b, n // page], np.arange(n % page, page)
            cache["k"][at][:, t] = 0x7F
            for i in t:
                cache["v"][at, :, i // 16, :, i % 16] = 0x7F
    got = _attend(B, ctx, torch, q, cache, table, lens, form)
    _attn_ok(got, want, mass)
    assert all((got[b] == 0).all() for b, n in enumerate(lens) if n == 0)
    assert (got == _attend(B, ctx, torch, q, cache, table, lens, form, dirty=False)).all()


def test_attention_pages_that_do_not_exist_and_lengths_out_of_range(env):
    B, ctx, torch = env
    rng = np.random.default_rng(7)
    heads, kv, dim, page = 6, 2, 64, 16
    cache = _filled(rng, 9, kv, page, dim)
    table = np.array([[0, 9, 2, -1], [-1, 1 << 30, 9, -(1 << 31)], [3, 4, 5, 6], [7, 8, 7, 8]], np.int32)
    q = _bits(rng, (4, heads, dim))
    for lens in ([64, 64, 1 << 30, -3], [40, 17, -(1 << 31), 61]):
        want, mass = OP.attn_paged(obf16.decode(q), cache, table, lens)
        got = _attend(B, ctx, torch, q, cache, table, lens)
        _attn_ok(got, want, mass)
        assert (got[1] == 0).all()                         # (not one page of it)


@pytest.mark.parametrize("page", [16, 64])
def test_attention_page_0_does_not_stand_in(env, page):
    """Entries that are no page, in a cache whose page 0 no sequence has and holds NaN, by codes and by exponents that are none."""
    B, ctx, torch = env
    rng = np.random.default_rng(11)
    heads, kv, dim = 4, 2, 128
    cache = _filled(rng, 5, kv, page, dim)
    cache["k"][0], cache["v"][0] = 0x7F, 0x7F
    cache["k_exps"][0], cache["v_exps"][0] = 255, 255
    table = np.array([[1, 5, 2], [-1, 3, 4], [-1, -1, -1]], np.int32)
    lens = [3 * page, 3 * page - 5, 2 * page]
    q = _bits(rng, (3, heads, dim))
    plain = {n: c.copy() for n, c in cache.items()}
    for n in plain:
        plain[n][0] = 120                                  # (nothing of it is looked at)
    want, mass = OP.attn_paged(obf16.decode(q), plain, table, lens)
    got = _attend(B, ctx, torch, q, cache, table, lens)
    _attn_ok(got, want, mass)
    assert (got[2] == 0).all()


@pytest.mark.parametrize("tokens", [40, 1500])
def test_attention_numbers_that_are_none(env, tokens):
    """A NaN among the keys of one head, among the values of a dim; scores of -inf throughout, of inf: the rows that the formula
    gives no number for, and no others."""
    B, ctx, torch = env
    rng = np.random.default_rng(8)
    heads, kv, dim, page = 4, 2, 64, 16
    table, pages = _deal(rng, [tokens] * 3, page)
    cache, q = _filled(rng, pages, kv, page, dim), _bits(rng, (3, heads, dim))
    want, mass = OP.attn_paged(obf16.decode(q), cache, table, [tokens] * 3)
    cache["k"][table[0, 1], 0, 3, 7] = 0x7F
    cache["v"][table[1, 2], 1, 0, 9, 5] = 0xFF
    q[2, 3, 5] = 0x7F80
    got = obf16.decode(_attend(B, ctx, torch, q, cache, table, [tokens] * 3))
    none = np.zeros(got.shape, bool)
    none[0, :2], none[1, 2:, 9], none[2, 3] = True, True, True
    assert np.isnan(got[none]).all()
    bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -12) * mass
    assert (np.abs(got - want)[~none] <= bound[~none]).all()
    # every score -inf: keys of one sign, one infinite number in q
    cache = _filled(rng, pages, kv, page, dim)
    cache["k"][..., 5] = 0x80 | 0x38
    got = obf16.decode(_attend(B, ctx, torch, q, cache, table, [tokens] * 3))
    assert np.isnan(got[2, 3]).all() and np.isfinite(got[2, :3]).all() and np.isfinite(got[:2]).all()


@pytest.mark.parametrize("scale", [0.01, 2.0])
def test_attention_scale_and_rising_scores(env, scale):
    """A maximum that keeps rising, weights far below it, exponents of blocks from tiny to huge."""
    B, ctx, torch = env
    rng = np.random.default_rng(9)
    n, page, dim = 1300, 16, 64
    table, pages = _deal(rng, [n], page)
    cache, q = _filled(rng, pages, 1, page, dim), _bits(rng, (1, 3, dim), 0.25)
    order = np.empty(pages, int)
    order[table[0]] = np.arange(table.shape[1])
    cache["k_exps"][table[0], 0] = 112 + np.arange(table.shape[1]) // 10   # keys grow by 2^8 along the sequence
    cache["v_exps"][:, 0] = rng.integers(100, 140, pages)
    want, mass = OP.attn_paged(obf16.decode(q), cache, table, [n], scale)
    got = obf16.decode(_attend(B, ctx, torch, q, cache, table, [n], scale=scale))
    # scores up to some hundreds: fp32's error of a score is (dim + 3) x 2^-24 of the sum of |q k| scale, which is below 1200 here,
    # and turns into as much of M
    k, _ = OP.tokens_of(cache, "k", table[0], n)
    size = scale * (np.abs(k[:, 0]) @ np.abs(obf16.decode(q)[0]).T).max()
    assert size < 12000
    bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -12 + 2 * (dim + 3) * 2.0 ** -24 * size) * mass
    assert (np.abs(got - want) <= bound).all()


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64)])
def test_attention_numbers_near_both_ends(env, dim, page):
    """Large queries on tiny keys and the other way round, values up to 2^96 and down to the smallest that can be stored."""
    B, ctx, torch = env
    rng = np.random.default_rng(10)
    lens = [40, 300]
    table, pages = _deal(rng, lens, page)
    cache, q = _filled(rng, pages, 4, page, dim), obf16.decode(_bits(rng, (2, 8, dim), 0.25))
    for head, (by_k, by_v) in enumerate([(-95, 94), (94, -117), (-95, -110), (0, -100)]):   # powers of two, exponents 1 to 216
        cache["k_exps"][:, head] = cache["k_exps"][:, head].astype(int) + by_k
        cache["v_exps"][:, head] = cache["v_exps"][:, head].astype(int) + by_v
        q[:, 2 * head:2 * head + 2] *= 2.0 ** -by_k
    q = TI.to_bf16_bits(q.astype(np.float32))
    assert cache["v_exps"].min() == 1 and np.abs(obf16.decode(q)).max() < 2.0 ** 96
    want, mass = OP.attn_paged(obf16.decode(q), cache, table, lens)
    got = obf16.decode(_attend(B, ctx, torch, q, cache, table, lens))
    # each value and each product with a weight may lose 2^-126, the sum of the weights is 1 or more, and the output once more
    tokens = np.array(lens)[:, None, None]
    bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -12) * mass + (2 * tokens + 1) * 2.0 ** -126
    assert (np.abs(got - want) <= bound).all()
    large = np.abs(want) > 2.0 ** -110                     # not lost in that
    assert large[:, :2].any() and large[:, 6:].any()


def test_attention_pages_shared_by_sequences_and_rows_apart(env):
    """A prefix's pages in every row of the table, a table and q with padding between rows."""
    B, ctx, torch = env
    rng = np.random.default_rng(10)
    page, dim, heads, kv, lens = 32, 128, 8, 2, [100, 70, 64, 33]
    cache = _filled(rng, 9, kv, page, dim)
    wide = np.array([[0, 1, 2, 3, 99], [0, 1, 4, 5, 99], [0, 1, 6, 6, 99], [0, 7, 8, 8, 99]], np.int32)
    q = _bits(rng, (4, heads + 2, dim))
    want, mass = OP.attn_paged(obf16.decode(q[:, :heads]), cache, wide[:, :4], lens)
    paged, tt, tq = _paged(B, torch, cache), _dev(torch, wide), _dev(torch, q)
    out = torch.zeros((4, heads, dim), dtype=torch.int16, device="cuda")
    size = B.attn_paged_scratch_bytes(4, heads, kv, dim, page, 4)
    scratch = torch.zeros(max(size, 1), dtype=torch.uint8, device="cuda")
    _run(ctx, torch, B.attn_paged_fp8(tq[:, :heads], paged, tt[:, :4], _dev(torch, np.array(lens, np.int32)), out, scratch), "hi")
    _attn_ok(_host(out), want, mass)


def test_caches_beyond_4_gib(env):
    """Pages whose bytes lie beyond 32 bits: appended to, and attended to."""
    B, ctx, torch = env
    rng = np.random.default_rng(11)
    kv, dim, page, pages = 8, 128, 128, 36000              # 4.7 GB of keys
    z = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")
    paged = B.PagedCache(z(pages, kv, page, dim), z(pages, kv, page // 16, dim, 16), z(pages, kv), z(pages, kv))
    table = np.array([[35999, 3, 35000]], np.int32)
    n = 300
    x, q = _bits(rng, (n, 2 * kv, dim)), _bits(rng, (1, 16, dim))
    tx, tt, tl = _dev(torch, x), _dev(torch, table), _dev(torch, np.array([n], np.int32))
    _run(ctx, torch, B.kv_append_fp8(tx[:, :kv], tx[:, kv:], _dev(torch, np.array([0, n], np.int32)), tl, tt, paged), "ptb")
    small = OP.append(obf16.decode(x[:, :kv]), obf16.decode(x[:, kv:]), [0, n], [n], np.array([[0, 1, 2]]), OP.empty_cache(3, kv, page, dim))
    _same([t[table[0].tolist()] for t in paged], small)
    touched = torch.zeros(pages, dtype=torch.bool, device="cuda")
    touched[table[0].tolist()] = True
    assert int(paged.k_exps[~touched].max()) == 0 and all(int(paged.k[i].max()) == 0 for i in (0, 1, 2, 2231, 3231, 35998))
    out = torch.zeros((1, 16, dim), dtype=torch.int16, device="cuda")
    scratch = z(max(B.attn_paged_scratch_bytes(1, 16, kv, dim, page, 3), 1))
    _run(ctx, torch, B.attn_paged_fp8(_dev(torch, q), paged, tt, tl, out, scratch), "hi")
    _attn_ok(_host(out), *OP.attn_paged(obf16.decode(q), small, np.array([[0, 1, 2]]), [n]))


def test_the_widest_rows(env):
    """As many heads as a token's row has room for."""
    B, ctx, torch = env
    rng = np.random.default_rng(22)
    x, freqs, at = _bits(rng, (3, 65536, 16)), (0.5 ** np.arange(8)).astype(np.float32), np.array([0, 70000, -9], np.int32)
    out = torch.zeros((3, 65536, 16), dtype=torch.int16, device="cuda")
    _run(ctx, torch, B.rope_bf16(_dev(torch, x), out, _dev(torch, freqs), _dev(torch, at), interleaved=True), "ptb")
    _rope_ok(_host(out), *OP.rope(obf16.decode(x), at, freqs, True))
    kv, dim, page, new, held = 700, 64, 16, [3, 0, 18], [20, 5, 1]
    cu, lens = np.concatenate([[0], np.cumsum(new)]).astype(np.int32), (np.array(new) + held).astype(np.int32)
    table, pages = _deal(rng, lens, page)
    cache = _filled(rng, pages, kv, page, dim)
    x, q = _bits(rng, (int(cu[-1]), 2 * kv, dim)), _bits(rng, (3, kv, dim), 0.5)
    paged, tx, tt = _paged(B, torch, cache), _dev(torch, x), _dev(torch, table)
    _run(ctx, torch, B.kv_append_fp8(tx[:, :kv], tx[:, kv:], _dev(torch, cu), _dev(torch, lens), tt, paged), "sliced")
    cache = OP.append(obf16.decode(x[:, :kv]), obf16.decode(x[:, kv:]), cu, lens, table, cache)
    _same(paged, cache)
    _attn_ok(_attend(B, ctx, torch, q, cache, table, lens), *OP.attn_paged(obf16.decode(q), cache, table, lens))
    # all query heads on one K/V head
    table, pages = _deal(rng, [300, 40], 32)
    cache, q = _filled(rng, pages, 1, 32, dim), _bits(rng, (2, 3001, dim), 0.5)
    _attn_ok(_attend(B, ctx, torch, q, cache, table, [300, 40]), *OP.attn_paged(obf16.decode(q), cache, table, [300, 40]))


# ---------------------------------------------------------------- together
def test_a_prompt_and_the_steps_behind_it(env):
    """As a serving job uses them: prompts are turned, attended to and appended; then steps turn their token's q, append its key and
    value and attend to the cache, with the lengths counted up on the device and the whole step captured into a graph."""
    B, ctx, torch = env
    rng = np.random.default_rng(12)
    heads, kv, dim, page, rot, steps = 8, 2, 64, 16, 32, 20
    first = [37, 1, 16]
    batch, total = len(first), sum(first)
    cu = np.concatenate([[0], np.cumsum(first)]).astype(np.int32)
    at = np.concatenate([np.arange(n) for n in first]).astype(np.int32)
    freqs, magnitude = B.rope_freqs(rot, factor=4.0, scaling="parts", context=64, turns=(1.0, 4.0), device="cuda")
    magnitude = float(np.float32(magnitude))               # (as the calls take it)
    table, pages = _deal(rng, [n + steps for n in first], page)
    cache = OP.empty_cache(pages, kv, page, dim)
    paged, tt, tcu = _paged(B, torch, cache), _dev(torch, table), _dev(torch, cu)
    lens = _dev(torch, np.array(first, np.int32))
    x = _bits(rng, (total, heads + 2 * kv, dim))
    tx = _dev(torch, x)
    turned, out = torch.zeros((total, heads + kv, dim), dtype=torch.int16, device="cuda"), torch.zeros((total, heads, dim), dtype=torch.int16, device="cuda")
    torch.cuda.synchronize()
    ctx.launch_native(B.rope_bf16(tx[:, :heads + kv], turned, freqs, _dev(torch, at), magnitude=magnitude))
    ctx.launch_native(B.attn_prompt_bf16(turned[:, :heads], turned[:, heads:], tx[:, heads + kv:], out, tcu))
    job = ctx.launch_ptb(B.kv_append_fp8(tx[:, heads:heads + kv], tx[:, heads + kv:], tcu, lens, tt, paged, freqs, magnitude=magnitude), 3)
    assert job.wait() == 3
    job.free()
    torch.cuda.synchronize()
    f64 = freqs.cpu().numpy()
    qk, mass = OP.rope(obf16.decode(x[:, :heads + kv]), at, f64, magnitude=magnitude)
    _rope_ok(_host(turned), qk, mass)
    qk = obf16.decode(_host(turned))
    _attn_ok(_host(out), *OS.attn_prompt(qk[:, :heads], qk[:, heads:], obf16.decode(x[:, heads + kv:]), cu))
    cache = OP.append(obf16.decode(x[:, heads:heads + kv]), obf16.decode(x[:, heads + kv:]), cu, first, table, cache, f64, None, False, magnitude)
    _same(paged, cache, "prompt")

    hi = ctx._streams[0]
    xs, q = torch.zeros((batch, heads + 2 * kv, dim), dtype=torch.int16, device="cuda"), torch.zeros((batch, heads, dim), dtype=torch.int16, device="cuda")
    o, one = torch.zeros((batch, heads, dim), dtype=torch.int16, device="cuda"), _dev(torch, np.arange(batch + 1).astype(np.int32))
    scratch = torch.zeros(max(B.attn_paged_scratch_bytes(batch, heads, kv, dim, page, table.shape[1]), 1), dtype=torch.uint8, device="cuda")
    places = lens.clone()
    kernels = [B.rope_bf16(xs[:, :heads], q, freqs, places, magnitude=magnitude),
               B.kv_append_fp8(xs[:, heads:heads + kv], xs[:, heads + kv:], one, lens, tt, paged, freqs, magnitude=magnitude),
               B.attn_paged_fp8(q, paged, tt, lens, o, scratch)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=hi):
        places.copy_(lens)
        lens.add_(1)
        for kern in kernels:
            ctx.launch_native(kern, hi=True)
    for step in range(steps):
        new = _bits(rng, (batch, heads + 2 * kv, dim))
        xs.copy_(_dev(torch, new))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        now = [n + step + 1 for n in first]
        want, mass = OP.rope(obf16.decode(new[:, :heads]), np.array(now) - 1, f64, magnitude=magnitude)
        _rope_ok(_host(q), want, mass)
        cache = OP.append(obf16.decode(new[:, heads:heads + kv]), obf16.decode(new[:, heads + kv:]), np.arange(batch + 1), now, table, cache, f64, None, False, magnitude)
        _same(paged, cache, f"step {step}")
        _attn_ok(_host(o), *OP.attn_paged(obf16.decode(_host(q)), cache, table, now))


def test_as_kernels_of_the_scheduler(env):
    """A best-effort client turns and appends in a loop, under configurations that the profiler tries; the high-priority one's
    requests turn, append and attend."""
    B, ctx, torch = env
    rng = np.random.default_rng(13)
    kv, heads, dim, page, n = 4, 8, 128, 32, 5000
    freqs = (10000.0 ** (-np.arange(64) / 64)).astype(np.float32)
    tf = _dev(torch, freqs)

    def side(n, seed):
        g = np.random.default_rng(seed)
        x = _bits(g, (n, heads + 2 * kv, dim))
        table, pages = _deal(g, [n], page)
        cache = OP.empty_cache(pages, kv, page, dim)
        return x, table, cache, _dev(torch, x), _dev(torch, table), _paged(B, torch, cache)
    x, table, cache, tx, tt, paged = side(n, 1)
    places, cu, lens = (_dev(torch, np.array(a, np.int32)) for a in (np.arange(n), [0, n], [n]))
    out = torch.zeros((n, heads + kv, dim), dtype=torch.int16, device="cuda")
    steps = [B.rope_bf16(tx[:, :heads + kv], out, tf, places), B.kv_append_fp8(tx[:, heads:heads + kv], tx[:, heads + kv:], cu, lens, tt, paged, tf)]
    hx, htable, hcache, htx, htt, hpaged = side(200, 2)
    hq, ho = torch.zeros((200, heads, dim), dtype=torch.int16, device="cuda"), torch.zeros((1, heads, dim), dtype=torch.int16, device="cuda")
    hcu, hlens = (_dev(torch, np.array(a, np.int32)) for a in ([0, 200], [200]))
    scratch = torch.zeros(max(B.attn_paged_scratch_bytes(1, heads, kv, dim, page, htable.shape[1]), 1), dtype=torch.uint8, device="cuda")
    request = [B.rope_bf16(htx[:, :heads], hq, tf, places[:200]), B.kv_append_fp8(htx[:, heads:heads + kv], htx[:, heads + kv:], hcu, hlens, htt, hpaged, tf),
               B.attn_paged_fp8(hq[199:], hpaged, htt, hlens, ho, scratch)]
    torch.cuda.synchronize()
    s = ctx.scheduler(profile_runs=2, threshold_ms=0.05)
    for kern in steps:
        s.submit_be(kern, loop=True)
    import time
    done, t0 = 0, time.time()
    while (done < 30 or s.stats()["be_kernels_done"] < 60) and time.time() - t0 < 30:
        s.submit_hi(request)
        while s.poll():
            pass
        done += 1
        time.sleep(0.002)
    stats = s.stats()
    s.close()
    torch.cuda.synchronize()
    assert done >= 30 and stats["be_kernels_done"] >= 60
    want, mass = OP.rope(obf16.decode(x[:, :heads + kv]), np.arange(n), freqs)
    _rope_ok(_host(out), want, mass)
    _same(paged, OP.append(obf16.decode(x[:, heads:heads + kv]), obf16.decode(x[:, heads + kv:]), [0, n], [n], table, cache, freqs), "best effort")
    hcache = OP.append(obf16.decode(hx[:, heads:heads + kv]), obf16.decode(hx[:, heads + kv:]), [0, 200], [200], htable, hcache, freqs)
    _same(hpaged, hcache, "high priority")
    _attn_ok(_host(ho), *OP.attn_paged(obf16.decode(_host(hq)[199:]), hcache, htable, [200]))
    rows = [ctx.profile_table(kern)[0] for kern in steps]
    assert all(rows) and sum(r["samples"] for t in rows for r in t) > 0
