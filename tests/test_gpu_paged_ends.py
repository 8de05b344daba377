"""GPU tests of the paged 8-bit cache at the ends of what it takes: turned keys of every size, memory beside the tensors, scores
of hundreds.  Helpers and tolerances are those of test_gpu_paged.py.

Codes and exponents are the oracle's.  The kernel's sines are off by 2e-14 (2^-45) at most, and where they are turned on from one
token to the next seven times that, 2^-42 of |x1| + |x2|; borders between codes lie 2^-4 of a number apart, so that one key of random
inputs is taken for another code with odds of 2^-37, and one of all 2^25 here and there with 2^-12."""
import numpy as np
import pytest

import tally_inputs as TI
from oracle import bf16 as obf16
from oracle import paged as OP
from test_gpu_paged import SENTINEL, _attend, _attn_ok, _bits, _cache, _deal, _dev, _filled, _host, _paged, _run, _same, env  # noqa: F401

pytestmark = pytest.mark.gpu

# new tokens of each sequence (dim, page) that take each way of appending: one wave a page, four waves a page, whole prompts
KINDS = [(1, 128, 128), (1, 64, 16), (5, 128, 128), (9, 64, 128), (16, 128, 16), (33, 128, 128), (40, 64, 64), (70, 64, 32)]


@pytest.mark.parametrize("form", ["hi", "ptb"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("new,dim,page", KINDS)
def test_append_turned_keys_next_to_borders_of_tiny_codes(env, new, dim, page, interleaved, form):
    """Keys that the turn takes from a border of two codes to beside it, in blocks of each of the lowest exponents: where numbers
    are subnormal in 32 bits that has to be known still when they are rounded to their code.  (The borders of a block lie within
    2^18.8 of one another, so a partner times 2^-24 to 2^-34 is above 2^-53 of the key: both sides' 64 bits see it.)"""
    B, ctx, torch = env
    rng = np.random.default_rng(new + dim)
    exps = np.arange(1, 13)
    n, kv, half = len(exps), 2, dim // 2
    borders = (OP.CODES[:126] + OP.CODES[1:127]) / 2
    # (bf16 has no numbers as small as the smallest border: the magnitude brings them down)
    magnitude = 2.0 ** -16
    x = np.zeros((n * new, 2 * kv, dim))
    sign = lambda s: rng.choice([-1.0, 1.0], s)
    for s, e in enumerate(exps):
        shape = (new, kv, dim)
        low = rng.random(shape) < 0.6                      # the borders of subnormal codes, and all others
        x[s * new:(s + 1) * new, :kv] = np.where(low, borders[rng.integers(0, 8, shape)], borders[rng.integers(0, 126, shape)]) * sign(shape) * 2.0 ** (e - 127.0) / magnitude
        x[s * new, :kv, 0] = 448 * 2.0 ** (e - 127.0) / magnitude   # the block's largest, alone in its pair
        x[s * new, :kv, 1 if interleaved else half] = 0
    x[:, kv:] = rng.standard_normal((n * new, kv, dim))
    bits = TI.to_bf16_bits(x.astype(np.float32))
    assert (obf16.decode(bits[:, :kv]) == x[:, :kv]).all()
    freqs = (2.0 ** -(24.0 + np.arange(half) % 11)).astype(np.float32)
    freqs[0] = 0
    held = rng.integers(0, page, n)
    cu, lens = (np.arange(n + 1) * new).astype(np.int32), (held + new).astype(np.int32)
    table, pages = _deal(rng, lens, page)
    cache = _cache(rng, pages, kv, page, dim, 1, 1)        # (held numbers do not raise the exponent)
    at = sign(n * new).astype(np.int32)
    want = OP.append(obf16.decode(bits[:, :kv]), obf16.decode(bits[:, kv:]), cu, lens, table, cache, freqs, at, interleaved, magnitude)
    assert set(exps) <= set(want["k_exps"].ravel())
    paged, tx = _paged(B, torch, cache), _dev(torch, bits)
    _run(ctx, torch, B.kv_append_fp8(tx[:, :kv], tx[:, kv:], _dev(torch, cu), _dev(torch, lens), _dev(torch, table), paged, _dev(torch, freqs),
                                     _dev(torch, at), interleaved, magnitude), form)
    _same(paged, want, form)


@pytest.mark.parametrize("magnitude", [1.0, 1.2, 64.0])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("new,dim,page", KINDS)
def test_append_turned_numbers_of_every_size(env, new, dim, page, interleaved, magnitude):
    """Keys from zeros to the largest, NaN and infinities among them, turned: what comes to 2^128 or more is infinite, stored as NaN and
    not counted for the block; what stays below is."""
    B, ctx, torch = env
    rng = np.random.default_rng(new + 2 * dim)
    tops = [0.0, 2.0 ** -133, 2.0 ** -126, 1.75, 448.0, 2.0 ** 120, 2.0 ** 127, 3.3e38]
    n, kv, half = len(tops), 2, dim // 2
    pair = (lambda i: (2 * i, 2 * i + 1)) if interleaved else (lambda i: (i, i + half))
    x = np.clip(rng.standard_normal((n * new, 2 * kv, dim)) / 2, -1, 1)
    for s, top in enumerate(tops):
        x[s * new:(s + 1) * new] *= top
        x[s * new, :, pair(3)[0]] = x[s * new, :, pair(3)[1]] = top   # (turned, one of them grows and one falls)
    bits = TI.to_bf16_bits(x.astype(np.float32))
    for s, (head, d, b) in enumerate(((0, 7, 0x7F80), (1, 9, 0xFF80), (0, dim - 1, 0x7FC0), (1, 0, 0xFFC0))):
        bits[(2 * s + 1) * new - 1, head, d] = b           # the last token of every other sequence
        bits[(2 * s + 1) * new - 1, kv + head, d] = b
    freqs = (0.9 ** np.arange(half)).astype(np.float32)
    held = rng.integers(0, page, n)
    cu, lens = (np.arange(n + 1) * new).astype(np.int32), (held + new).astype(np.int32)
    table, pages = _deal(rng, lens, page)
    cache = _cache(rng, pages, kv, page, dim, 1, 130)
    by = float(np.float32(magnitude))
    with np.errstate(invalid="ignore", over="ignore"):
        want = OP.append(obf16.decode(bits[:, :kv]), obf16.decode(bits[:, kv:]), cu, lens, table, cache, freqs, None, interleaved, by)
        turned = np.abs(OP.rope(obf16.decode(bits[:, :kv]), np.concatenate([np.arange(h, h + new) for h in held]), freqs, interleaved, False, by)[0])
    assert ((turned >= 2.0 ** 128) & np.isfinite(turned)).any()
    paged, tx = _paged(B, torch, cache), _dev(torch, bits)
    _run(ctx, torch, B.kv_append_fp8(tx[:, :kv], tx[:, kv:], _dev(torch, cu), _dev(torch, lens), _dev(torch, table), paged, _dev(torch, freqs),
                                     interleaved=interleaved, magnitude=magnitude), "hi")
    _same(paged, want)


def test_questions_about_calls_that_are_refused(env):
    """The profiler's records of descriptors that no launch takes, of sizes that stand below a division among them: there are none."""
    B, ctx, torch = env
    import ctypes as C
    ctx.profile_reset()
    args = dict(k=4096, v=4096, cu_seqlens=4096, lens=4096, table=4096, k_pages=4096, v_pages=4096, k_exps=4096, v_exps=4096, total=1000, n_seqs=3, kv_heads=2,
                dim=64, page=16, n_pages=100, seq_pages=40)
    for bad in (dict(dim=0), dict(dim=2048), dict(page=0), dict(n_seqs=0), dict(total=0), dict(k=None)):
        a = B.KvAppendArgs(**dict(args, **bad))
        with pytest.raises(B.TallyError):
            B.logical_grid(B.K_KV_APPEND_FP8, a)
        kern = B.Kernel.__new__(B.Kernel)
        kern.args, kern.desc = a, B.KernelDesc(B.K_KV_APPEND_FP8, B.Dim3(10, 1, 1), B.Dim3(256, 1, 1), C.addressof(a), C.sizeof(a))
        assert ctx.lookup_config(kern) is None and ctx.profile_table(kern) == ([], -1)
        with pytest.raises(B.TallyError):
            ctx.launch_native(kern)


def test_measurements_of_blocks_with_different_work_are_kept_apart(env):
    """Calls whose grids are equal and whose blocks' work is not: how many tokens or heads a block goes through, what is turned
    and from what.  One call's records and choice are not another's."""
    B, ctx, torch = env
    z = lambda *s: torch.zeros(s, dtype=torch.int16, device="cuda")

    def rope(total, dim, rot, **how):
        x = z(total, 8, dim)
        return B.rope_bf16(x, x, torch.zeros(rot // 2, device="cuda"), torch.zeros(total, dtype=torch.int32, device="cuda"), **how)

    def append(total, rot, kv=8, dim=128, page=16, at=False, **how):
        x, cache = z(total, 2 * kv, dim), B.PagedCache.empty(-(-total // page), kv, page, dim)
        ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
        return B.kv_append_fp8(x[:, :kv], x[:, kv:], ints(0, total), ints(total), torch.arange(len(cache.k), dtype=torch.int32, device="cuda")[None],
                               cache, torch.zeros(rot // 2, device="cuda") if rot else None,
                               torch.zeros(total, dtype=torch.int32, device="cuda") if at else None, **how)
    # 1500 blocks of a token, and 3000 tokens in blocks of two; a head a wave, and two
    calls = [[rope(1500, 64, 64), rope(3000, 64, 64), rope(1500, 64, 32), rope(1500, 64, 64, interleaved=True), rope(1500, 128, 64)],
             [append(480, 128), append(480, 0), append(480, 64), append(480, 128, interleaved=True), append(480, 128, at=True)],
             [append(8192 + 16, 128), append(4112 - 16, 128), append(8192 + 16, 0)]]
    ctx.profile_reset()
    torch.cuda.synchronize()
    for same in calls:
        for i, kern in enumerate(same):
            assert kern.desc.grid.x == same[0].desc.grid.x
            for later in same[i:]:
                assert ctx.profile_table(later) == ([], -1) and ctx.lookup_config(later) is None
            ctx.profile(kern, [(B.CFG_PTB, 4, 1), (B.CFG_SLICED, 1 + i, 1)], runs=1)
        assert [ctx.profile_table(k)[0][1]["param"] for k in same] == [1 + i for i in range(len(same))]
    assert len(ctx.profile_table(append(475, 128))[0]) == 2   # (a few tokens fewer: the same blocks)
    ctx.profile_reset()


def _steep(rng, pattern, n):
    """Scores of n tokens for the first query head: hundreds, in an order that a running maximum can go wrong with."""
    low = rng.uniform(-200, -150, n)
    if pattern == "rising":
        return np.linspace(-300, 300, n)
    if pattern == "falling":
        return np.linspace(300, -300, n)
    if pattern == "steps":                                 # from one tile of 32 tokens to the next, up and far down
        return np.array([200.0, 250, 300, -175, -200])[np.arange(n) // 32 % 5]
    at = {"first": [2], "last": [n - 2], "one wave": [n // 256 * 128 + 64 + 7], "ends": [1, n - 1], "a tile": range(n - 40, n - 30)}[pattern]
    low[list(at)] = 300
    return low


@pytest.mark.parametrize("pattern", ["first", "last", "one wave", "ends", "a tile", "steps", "rising", "falling"])
@pytest.mark.parametrize("n", [400, 1300, 4000])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64)])
def test_attention_scores_of_hundreds(env, dim, page, n, pattern):
    """Scores from -300 to 300: weights that vanish beside a later maximum, waves and parts whose state as a whole does.  400 tokens are
    one part, 1300 six parts (a wave merges a row), 4000 sixteen (a workgroup does)."""
    B, ctx, torch = env
    rng = np.random.default_rng(n + dim)
    heads, scale = 4, 0.125
    table, pages = _deal(rng, [n], page)
    cache = _filled(rng, pages, 1, page, dim)
    assert (B.attn_paged_scratch_bytes(1, heads, 1, dim, page, table.shape[1]) == 0) == (n == 400)
    q = rng.uniform(0.5, 1.5, (1, heads, dim)) * rng.choice([-1.0, 1.0], (1, heads, dim))
    q[0, 1], q[0, 2] = -q[0, 0], q[0, 0] * 0.25            # the other way round, and less steep; the last one is its own
    bits = TI.to_bf16_bits(q.astype(np.float32))
    q = obf16.decode(bits)
    k = _steep(rng, pattern, n)[:, None] * np.sign(q[0, 0]) / (scale * np.abs(q[0, 0]).sum()) * rng.uniform(0.75, 1.25, (n, dim))
    # (the pages are then filled as an append fills them)
    x = TI.to_bf16_bits(np.stack([k, rng.standard_normal((n, dim))], 1).astype(np.float32))
    x = obf16.decode(x)
    cache = OP.append(x[:, :1], x[:, 1:], [0, n], [n], table, cache)
    want, mass = OP.attn_paged(q, cache, table, [n], scale)
    codes, _ = OP.tokens_of(cache, "k", table[0], n)
    scores = scale * codes[:, 0] @ q[0].T
    size = scale * (np.abs(codes[:, 0]) @ np.abs(q[0]).T).max()
    assert scores[:, 0].max() > 250 and np.ptp(scores[:, 0]) > 400 and size < 400
    got = _attend(B, ctx, torch, bits, cache, table, [n], scale=scale)
    # fp32's error of a score, dim + 3 roundings of at most `size`, is one of its weight; of the sums too
    bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -12 + 2 * (dim + 3) * 2.0 ** -24 * size) * mass
    err = np.abs(obf16.decode(got) - want)
    assert (err <= bound).all(), f"worst {(err / bound).max():.2f} bounds"


def _amid(torch, a, fill, beside=1 << 16):
    """A tensor in the middle of a larger one that is filled otherwise; and that one."""
    t = _dev(torch, a)
    n = beside // t.element_size()
    whole = torch.full((t.numel() + 2 * n,), fill, dtype=t.dtype, device="cuda")
    whole[n:-n] = t.view(-1)
    return whole[n:-n].view(t.shape), whole


def _beside_is(whole, fill, beside=1 << 16):
    n = beside // whole.element_size()
    return bool((whole[:n] == fill).all()) and bool((whole[-n:] == fill).all())


# tokens of each sequence, so that a page is one wave's, four waves', or all its pieces have a wave; the last two with two heads a wave
PLACES = [(1, 64, 16, 2), (1, 128, 128, 3), (5, 128, 128, 2), (9, 64, 128, 3), (7, 128, 64, 1), (19, 64, 16, 3), (70, 64, 64, 2), (150, 128, 128, 2), (67, 128, 32, 5),
          (800, 128, 16, 7), (1500, 64, 64, 7)]


@pytest.mark.parametrize("form", ["hi", "be", "sliced", "ptb"])
@pytest.mark.parametrize("new,dim,page,kv", PLACES)
def test_append_touches_its_places_alone(env, new, dim, page, kv, form):
    """Pages that do not exist, places before the first and behind the last page, lengths and ends of sequences out of range: what has no place
    is not stored, and the bytes before and behind the pages and exponents stay as they are.  Around k and v there are NaN."""
    B, ctx, torch = env
    rng = np.random.default_rng(new + page)
    n, wide = 13, -(-new // page) + 2
    cu = (np.arange(n + 1) * new).astype(np.int32)
    total = int(cu[-1])
    cu[0], cu[-1] = -9, 1 << 30
    lens = np.full(n, new, np.int64) + rng.integers(0, page, n)
    table = np.full((n, wide), -1, np.int64)
    ids = iter(rng.permutation(n * wide))
    for s in range(n):
        table[s] = [next(ids) for _ in range(wide)]
    pages, at = n * wide + 2, (lens - 1) // page            # (two that are nobody's; the last token's)
    for s, none in ((1, -1), (2, pages), (3, 1 << 30), (4, -(1 << 31)), (5, (1 << 31) - 1)):
        table[s, at[s]] = none
    lens[6], lens[7], lens[8] = new // 2, wide * page + new // 2, 0
    lens[9], lens[10], lens[11] = -7, 1 << 30, (1 << 31) - 1
    lens, table = lens.astype(np.int32), table.astype(np.int32)
    cache, x = _cache(rng, pages, kv, page, dim), _bits(rng, (total, 2 * kv, dim))
    freqs = (10000.0 ** (-np.arange(dim // 2) / (dim // 2))).astype(np.float32)
    places = rng.integers(0, 1 << 20, total).astype(np.int32) if form in ("be", "ptb") else None
    parts = {m: _amid(torch, cache[m], 0x5A) for m in ("k", "v", "k_exps", "v_exps")}
    paged = B.PagedCache(*(parts[m][0] for m in ("k", "v", "k_exps", "v_exps")))
    tx, whole_x = _amid(torch, x, 0x7FC0)
    tt, _ = _amid(torch, table, pages - 1)
    kern = B.kv_append_fp8(tx[:, :kv], tx[:, kv:], _dev(torch, cu), _dev(torch, lens), tt, paged, _dev(torch, freqs),
                           None if places is None else _dev(torch, places), interleaved=kv % 2 == 0)
    want = OP.append(obf16.decode(x[:, :kv]), obf16.decode(x[:, kv:]), cu, lens, table, cache, freqs, places, kv % 2 == 0)
    assert all((want["k"][p] == cache["k"][p]).all() for p in (pages - 2, pages - 1)) and (want["k"] != cache["k"]).any()
    _run(ctx, torch, kern, form)
    _same(paged, want, form)
    assert all(_beside_is(parts[m][1], 0x5A) for m in parts) and _beside_is(whole_x, 0x7FC0)
    assert (_host(tx) == x).all() and (_host(tt) == table).all()


@pytest.mark.parametrize("form", ["hi", "ptb"])
@pytest.mark.parametrize("new,dim,page,kv", PLACES[::2])
def test_append_whatever_the_indexes_hold(env, new, dim, page, kv, form):
    """Ends of sequences in no order, any lengths, any table, of which only the pages of the pool may be written."""
    B, ctx, torch = env
    rng = np.random.default_rng(new + 3 * page)
    n, wide, pages = 13, 5, 30
    total = n * new
    cache, x = _cache(rng, pages, kv, page, dim), _bits(rng, (total, 2 * kv, dim))
    parts = {m: _amid(torch, cache[m], 0x5A) for m in ("k", "v", "k_exps", "v_exps")}
    paged = B.PagedCache(*(parts[m][0] for m in ("k", "v", "k_exps", "v_exps")))
    tx, _ = _amid(torch, x, 0x7FC0)
    any_int = lambda shape, most: np.where(rng.random(shape) < 0.3, rng.integers(-(1 << 31), 1 << 31, shape), rng.integers(-3, most, shape)).astype(np.int32)
    for _ in range(3):
        cu, lens, table = any_int(n + 1, total + 3), any_int(n, wide * page + 3), any_int((n, wide), pages + 3)
        _run(ctx, torch, B.kv_append_fp8(tx[:, :kv], tx[:, kv:], _dev(torch, cu), _dev(torch, lens), _dev(torch, table), paged), form)
        assert all(_beside_is(parts[m][1], 0x5A) for m in parts) and (_host(tx) == x).all()


@pytest.mark.parametrize("lens,heads,kv,dim,page,more", [
    ([1300], 3, 1, 64, 16, 0), ([4000], 2, 2, 128, 64, 0), ([900, 33], 40, 1, 128, 16, 0), ([0, 5, 3000], 28, 4, 128, 32, 3), ([700 + i for i in range(40)], 8, 8, 64, 64, 40),
    ([40, 300], 12, 12, 64, 16, 400)])
def test_attention_stays_within_its_scratch(env, lens, heads, kv, dim, page, more):
    """Scratch of the very size that is asked for, pages and table in the middle of others: nothing beside them is written or counts."""
    B, ctx, torch = env
    rng = np.random.default_rng(len(lens) + heads)
    table, pages = _deal(rng, lens, page, more=more)
    cache, q = _filled(rng, pages, kv, page, dim), _bits(rng, (len(lens), heads, dim))
    size = B.attn_paged_scratch_bytes(len(lens), heads, kv, dim, page, table.shape[1])
    assert size > 0
    scratch, whole = _amid(torch, np.full(size, 0xFF, np.uint8), 0x5A)
    paged = B.PagedCache(*(_amid(torch, cache[m], f)[0] for m, f in (("k", 0x7F), ("v", 0x7F), ("k_exps", 255), ("v_exps", 255))))
    out, whole_out = _amid(torch, np.full((len(lens), heads, dim), SENTINEL, np.uint16), SENTINEL)
    _run(ctx, torch, B.attn_paged_fp8(_amid(torch, q, 0x7FC0)[0], paged, _amid(torch, table, 0)[0], _dev(torch, np.array(lens, np.int32)), out, scratch), "hi")
    _attn_ok(_host(out), *OP.attn_paged(obf16.decode(q), cache, table, lens))
    assert _beside_is(whole, 0x5A) and _beside_is(whole_out, SENTINEL)


@pytest.mark.parametrize("heads,kv,dim,page,width", [(4, 1, 64, 16, 4000), (16, 8, 128, 64, 700), (6, 2, 128, 32, 2000)])
def test_a_captured_call_as_lengths_change(env, heads, kv, dim, page, width):
    """A graph of an append and the attention behind it, captured once with a table for the longest, replayed as the lengths on the device go from
    nothing to all of it and back: in as many parts as there are then, merged by a wave or a workgroup a row, with eager calls between."""
    B, ctx, torch = env
    rng = np.random.default_rng(width)
    batch, new = 3, 2
    table, pages = _deal(rng, [width] * batch, page)
    cache = _filled(rng, pages, kv, page, dim)
    paged, tt = _paged(B, torch, cache), _dev(torch, table)
    x, q = _bits(rng, (batch * new, 2 * kv, dim)), _bits(rng, (batch, heads, dim))
    tx, tq, cu = _dev(torch, x), _dev(torch, q), _dev(torch, (np.arange(batch + 1) * new).astype(np.int32))
    lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
    out = torch.zeros((batch, heads, dim), dtype=torch.int16, device="cuda")
    scratch = torch.full((B.attn_paged_scratch_bytes(batch, heads, kv, dim, page, table.shape[1]),), 0xFF, dtype=torch.uint8, device="cuda")
    assert scratch.numel() > 0
    kernels = [B.kv_append_fp8(tx[:, :kv], tx[:, kv:], cu, lens, tt, paged), B.attn_paged_fp8(tq, paged, tt, lens, out, scratch)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=ctx._streams[0]):
        for kern in kernels:
            ctx.launch_native(kern, hi=True)
    # (an append of two tokens counts as the last two: with fewer the first ones have no place)
    for now in ([0, 0, 0], [1, 0, 2], [130, width, 7], [width, width, width], [width // 2, 300, 129], [2, 0, width - 1], [width, 1, 0]):
        lens.copy_(_dev(torch, np.array(now, np.int32)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        cache = OP.append(obf16.decode(x[:, :kv]), obf16.decode(x[:, kv:]), np.arange(batch + 1) * new, now, table, cache)
        _same(paged, cache, str(now))
        got = _host(out).copy()
        _attn_ok(got, *OP.attn_paged(obf16.decode(q), cache, table, now))
        out.fill_(0)
        scratch.fill_(0xFF)
        _run(ctx, torch, kernels[1], "be")
        assert (_host(out) == got).all()


def test_two_calls_at_once(env):
    """On both streams together, a scratch each: appends to different sequences of one cache, and attention over it."""
    B, ctx, torch = env
    rng = np.random.default_rng(31)
    heads, kv, dim, page, n = 16, 4, 128, 32, 3000
    table, pages = _deal(rng, [n, n], page)
    cache = _filled(rng, pages, kv, page, dim)
    paged = _paged(B, torch, cache)
    x, q = [_bits(rng, (n, 2 * kv, dim)) for _ in range(2)], _bits(rng, (2, heads, dim))
    cu, tq = _dev(torch, np.array([0, n], np.int32)), _dev(torch, q)
    tl, tt = _dev(torch, np.array([n, n], np.int32)), _dev(torch, table)
    out = torch.zeros((2, heads, dim), dtype=torch.int16, device="cuda")
    size = B.attn_paged_scratch_bytes(1, heads, kv, dim, page, table.shape[1])
    assert size > 0
    appends, attends = [], []
    for i in range(2):
        tx = _dev(torch, x[i])
        appends.append(B.kv_append_fp8(tx[:, :kv], tx[:, kv:], cu, tl[i:i + 1], tt[i:i + 1], paged))
        attends.append(B.attn_paged_fp8(tq[i:i + 1], paged, tt[i:i + 1], tl[i:i + 1], out[i:i + 1], torch.zeros(size, dtype=torch.uint8, device="cuda")))
        cache = OP.append(obf16.decode(x[i][:, :kv]), obf16.decode(x[i][:, kv:]), [0, n], [n], table[i:i + 1], cache)
    want, mass = OP.attn_paged(obf16.decode(q), cache, table, [n, n])
    first = None
    for _ in range(20):
        out.fill_(0)
        torch.cuda.synchronize()
        for both in (appends, attends):
            for i in range(2):
                ctx.launch_native(both[i], hi=i == 0)
        torch.cuda.synchronize()
        got = _host(out).copy()
        first = got if first is None else first
        assert (got == first).all()
    _same(paged, cache)
    _attn_ok(first, want, mass)
