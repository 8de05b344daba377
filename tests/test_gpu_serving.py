"""GPU parity of the serving operators (prompt attention, shared-prefix attention, 4-bit products)
against their fp64 statements, in every launch form, at the sizes and masks where they can go wrong.

Tolerances, all of them from the arithmetic.  bf16 rounds by at most 2^-8 of a value.
  attention: the output is rounded once, and each p once before the second product:
    |d| <= 2^-8 |want| + (2^-8 + 2^-12) M, with M = sum p |v| / sum p.  2^-12 covers fp32: scores of magnitude s
    have an absolute error below (dim + 2) s 2^-24 (130 x 40 x 2^-24 < 2^-11.6 only beyond s = 40; inputs here stay
    below s = 20) and sums of up to 4096 terms at most 2^-12 of M, in practice far less.
  4-bit products: rounded once; a group's sums and the sum over groups are fp32 chains of at most 2 k + 300
    additions of terms whose magnitudes sum to M = sum (256 + code + zero) |x| s >= what is added:
    |d| <= 2^-8 |want| + (2 k + 300) 2^-24 M.
"""
import numpy as np
import pytest

import tally_inputs as TI
from oracle import bf16 as obf16
from oracle import serving as OS

pytestmark = pytest.mark.gpu
SENTINEL = 0x7ABC                                          # a bf16 that no output is


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
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda()


def _host(t):
    return t.cpu().numpy().view(np.uint16)


def _attn_ok(got_bits, want, mass):
    got = obf16.decode(got_bits)
    bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -12) * mass
    assert np.isfinite(got).all()
    err = np.abs(got - want)
    assert (err <= bound).all(), f"{(err > bound).sum()} of {err.size} off; worst {(err / np.maximum(bound, 1e-30)).max():.2f} bounds"


def _run(ctx, torch, kernel, form):
    """The whole kernel in one of its forms."""
    if form == "hi" or form == "be":
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


# ---------------------------------------------------------------- whole prompts
def _prompt(torch, seed, edges, total, heads, kv_heads, dim, scale=1.0):
    rng = np.random.default_rng(seed)
    q, k, v = (_bits(rng, (total, h, dim), scale) for h in (heads, kv_heads, kv_heads))
    cu = torch.tensor(edges, dtype=torch.int32, device="cuda")
    return q, k, v, cu


CASES = [
    ([0, 1], 1, 1, 1, 128), ([0, 2], 2, 2, 1, 64), ([0, 31], 31, 1, 1, 128), ([0, 32], 32, 3, 3, 64), ([0, 33], 33, 2, 2, 128),
    ([0, 63], 63, 1, 1, 64), ([0, 64], 64, 2, 1, 128), ([0, 65], 65, 1, 1, 128), ([0, 127], 127, 1, 1, 64),
    ([0, 128], 128, 1, 1, 128), ([0, 129], 129, 2, 1, 128), ([0, 300], 300, 7, 1, 128), ([0, 300], 301, 4, 2, 64),
    # packed: empty sequences, single tokens, starts away from any tile, rows before and behind them
    ([0, 1, 1, 2, 66, 66, 193], 193, 4, 2, 128), ([5, 5, 20, 148, 150], 160, 3, 1, 64),
    ([0, 127, 128, 129, 257, 258], 300, 2, 2, 128), ([100, 229], 400, 1, 1, 128),
    # as many heads as dies, and more
    ([0, 300, 301, 450], 450, 8, 2, 64), ([0, 130, 500], 500, 16, 4, 128), ([3, 140], 150, 24, 24, 64),
]


@pytest.mark.parametrize("form", ["hi", "be", "sliced", "ptb"])
@pytest.mark.parametrize("edges,total,heads,kv_heads,dim", CASES)
def test_prompt_attention(env, edges, total, heads, kv_heads, dim, form):
    B, ctx, torch = env
    q, k, v, cu = _prompt(torch, total + dim, edges, total, heads, kv_heads, dim)
    out = torch.full((total, heads, dim), SENTINEL, dtype=torch.int16, device="cuda")
    kern = B.attn_prompt_bf16(_dev(torch, q), _dev(torch, k), _dev(torch, v), out, cu)
    torch.cuda.synchronize()
    _run(ctx, torch, kern, form)
    want, mass = OS.attn_prompt(obf16.decode(q), obf16.decode(k), obf16.decode(v), edges)
    mine = ~np.isnan(want[:, 0, 0])
    got = _host(out)
    _attn_ok(got[mine], want[mine], mass[mine])
    assert (got[~mine] == SENTINEL).all()                  # rows of no sequence stay as they were


@pytest.mark.parametrize("dim", [64, 128])
def test_prompt_forms_give_the_same_bits(env, dim):
    B, ctx, torch = env
    edges = [0, 700, 701, 1500]
    q, k, v, cu = _prompt(torch, 3, edges, 1500, 4, 2, dim)
    q, k, v = (_dev(torch, t) for t in (q, k, v))
    outs = []
    for form in ("hi", "be", "sliced", "ptb", "ptb"):
        out = torch.zeros_like(q)
        kern = B.attn_prompt_bf16(q, k, v, out, cu)
        torch.cuda.synchronize()
        _run(ctx, torch, kern, form)
        outs.append(_host(out))
    assert all((o == outs[0]).all() for o in outs)


@pytest.mark.parametrize("scale", [0.02, 1.5])
def test_prompt_scale_and_large_scores(env, scale):
    """A maximum that keeps rising (scores up to some hundreds): rescaling, and weights far below it."""
    B, ctx, torch = env
    total, dim = 260, 64
    rng = np.random.default_rng(8)
    ramp = np.linspace(0.1, 2.0, total)[:, None, None]
    q, k, v = _bits(rng, (total, 2, dim)), TI.to_bf16_bits((rng.standard_normal((total, 1, dim)) * ramp).astype(np.float32)), _bits(rng, (total, 1, dim))
    out = torch.zeros((total, 2, dim), dtype=torch.int16, device="cuda")
    cu = torch.tensor([0, total], dtype=torch.int32, device="cuda")
    kern = B.attn_prompt_bf16(_dev(torch, q), _dev(torch, k), _dev(torch, v), out, cu, scale=scale)
    torch.cuda.synchronize()
    _run(ctx, torch, kern, "hi")
    want, mass = OS.attn_prompt(obf16.decode(q), obf16.decode(k), obf16.decode(v), [0, total], scale)
    _attn_ok(_host(out), want, mass)


@pytest.mark.parametrize("dim,scale,reach", [(64, 1.5, 3.0), (128, 0.8, 6.0), (64, 20.0, 3.0)])
def test_prompt_scores_of_hundreds_and_thousands(env, dim, scale, reach):
    """A maximum that keeps rising over scores of magnitude S, up to some thousands.  A score's products and sums are off by
    (dim + 2) S 2^-24, p by as much of itself, and so are numerator and denominator, each by that much of M."""
    B, ctx, torch = env
    total = 520
    rng = np.random.default_rng(dim)
    ramp = np.linspace(0.05, reach, total)[:, None, None]
    q, v = _bits(rng, (total, 4, dim)), _bits(rng, (total, 2, dim))
    k = TI.to_bf16_bits((rng.standard_normal((total, 2, dim)) * ramp).astype(np.float32))
    out = torch.zeros((total, 4, dim), dtype=torch.int16, device="cuda")
    cu = torch.tensor([0, 200, total], dtype=torch.int32, device="cuda")
    kern = B.attn_prompt_bf16(_dev(torch, q), _dev(torch, k), _dev(torch, v), out, cu, scale=scale)
    torch.cuda.synchronize()
    _run(ctx, torch, kern, "hi")
    qd, kd = obf16.decode(q), obf16.decode(k)
    want, mass = OS.attn_prompt(qd, kd, obf16.decode(v), [0, 200, total], scale)
    S = scale * np.abs(qd).sum(-1).max() * np.abs(kd).max()   # (at least sum |q k| of any pair)
    S = min(S, scale * np.sqrt((qd ** 2).sum(-1).max() * (kd ** 2).sum(-1).max()))
    bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -12 + 2 * (dim + 2) * S * 2.0 ** -24) * mass
    assert S > 100
    err = np.abs(obf16.decode(_host(out)) - want)
    assert (err <= bound).all(), (err / bound).max()


def test_prompt_strided_views_of_one_buffer(env):
    """q, k and v of a fused projection's padded output, out a view with padding of its own."""
    B, ctx, torch = env
    total, heads, kv, dim = 200, 6, 2, 128
    rng = np.random.default_rng(4)
    whole = _bits(rng, (total, heads + 2 * kv + 1, dim))
    buf = _dev(torch, whole)
    out = torch.full((total, heads + 3, dim), SENTINEL, dtype=torch.int16, device="cuda")
    kern = B.attn_prompt_bf16(buf[:, :heads], buf[:, heads:heads + kv], buf[:, heads + kv:heads + 2 * kv], out[:, 1:1 + heads],
                              torch.tensor([0, 50, total], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    _run(ctx, torch, kern, "hi")
    w = obf16.decode(whole)
    want, mass = OS.attn_prompt(w[:, :heads], w[:, heads:heads + kv], w[:, heads + kv:heads + 2 * kv], [0, 50, total])
    got = _host(out)
    _attn_ok(got[:, 1:1 + heads], want, mass)
    assert (got[:, 0] == SENTINEL).all() and (got[:, 1 + heads:] == SENTINEL).all()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("poison", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("where", [0, 17, 40, 63, 64, 100, 129])
def test_prompt_rows_do_not_see_what_is_hidden_from_them(env, where, poison, dim):
    """K and V of one token are no numbers: rows before it, and other sequences, are what they are without
    it; rows from it on are not finite where the definition's are not."""
    B, ctx, torch = env
    edges, total = [0, 130, 190], 195
    q, k, v, cu = _prompt(torch, where, edges, total, 2, 1, dim)
    bad = TI.to_bf16_bits(np.float32([poison]))[0]
    want, mass = OS.attn_prompt(obf16.decode(q), obf16.decode(k), obf16.decode(v), edges)
    for keys in (False, True):
        k2, v2 = k.copy(), v.copy()
        v2[where, 0, 3:9] = bad
        v2[192:] = bad                                     # rows behind the last sequence
        k2[192:] = bad
        if keys:
            k2[where] = bad
        out = torch.zeros((total, 2, dim), dtype=torch.int16, device="cuda")
        kern = B.attn_prompt_bf16(_dev(torch, q), _dev(torch, k2), _dev(torch, v2), out, cu)
        torch.cuda.synchronize()
        _run(ctx, torch, kern, "hi")
        got = _host(out)
        fine = np.r_[0:where, 130:190]
        _attn_ok(got[fine], want[fine], mass[fine])
        seen = obf16.decode(got[where:130])
        if not keys:
            hit = seen[:, :, 3:9]
            assert np.isnan(hit).all() if np.isnan(poison) else (hit == poison).all()
            rest = np.r_[0:3, 9:dim]
            _attn_ok(got[where:130][:, :, rest], want[where:130][:, :, rest], mass[where:130][:, :, rest])
        else:
            # (q has both signs, so a key of infinities has a score of NaN as well: the whole row is NaN)
            assert np.isnan(seen).all()


@pytest.mark.parametrize("seqs", [62, 63, 64, 65, 700, 3969, 3970, 5000])
def test_prompt_many_sequences(env, seqs):
    """The search for a block's sequence, with one, two and three rounds of 64 candidates."""
    B, ctx, torch = env
    rng = np.random.default_rng(seqs)
    lens = rng.integers(0, 4, seqs)
    lens[rng.integers(0, seqs)] = 140
    edges = np.concatenate([[0], np.cumsum(lens)]).astype(int).tolist()
    total = edges[-1]
    q, k, v, cu = _prompt(torch, seqs, edges, total, 1, 1, 64)
    out = torch.full((total, 1, 64), SENTINEL, dtype=torch.int16, device="cuda")
    kern = B.attn_prompt_bf16(_dev(torch, q), _dev(torch, k), _dev(torch, v), out, cu)
    torch.cuda.synchronize()
    _run(ctx, torch, kern, "hi")
    want, mass = OS.attn_prompt(obf16.decode(q), obf16.decode(k), obf16.decode(v), edges)
    _attn_ok(_host(out), want, mass)


@pytest.mark.parametrize("edges", [[-5, 40, 20, 100, 9000], [90, 10], [0, 0, 0], [200, 300], [-9, -1, 7]])
def test_prompt_with_edges_that_make_no_sense_stays_in_bounds(env, edges):
    """Entries outside [0, total] count as its ends and an end before its start as an empty sequence (the
    kernel clamps what it reads); neighbours of the tensors stay as they were."""
    B, ctx, torch = env
    total, dim = 100, 64
    room = torch.full((3 * total, 2, dim), SENTINEL, dtype=torch.int16, device="cuda")
    x = _dev(torch, _bits(np.random.default_rng(1), (total, 2, dim)))
    kern = B.attn_prompt_bf16(x, x, x, room[total:2 * total], torch.tensor(edges, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    _run(ctx, torch, kern, "hi")
    got = _host(room)
    assert (got[:total] == SENTINEL).all() and (got[2 * total:] == SENTINEL).all()
    assert np.isfinite(obf16.decode(got[total:2 * total])).all()


def test_prompt_offsets_beyond_32_bits(env):
    """Tokens so far apart that the last ones lie 4 GB and more behind the first."""
    B, ctx, torch = env
    total, ld, dim = 2200, 1 << 20, 64
    rng = np.random.default_rng(6)
    q, k, v = (_bits(rng, (total, 1, dim)) for _ in range(3))
    big = torch.empty(total * ld, dtype=torch.int16, device="cuda").view(total, ld // dim, dim)
    big[:, 0:1], big[:, 1:2], big[:, 2:3] = _dev(torch, q), _dev(torch, k), _dev(torch, v)
    kern = B.attn_prompt_bf16(big[:, 0:1], big[:, 1:2], big[:, 2:3], big[:, 3:4], torch.tensor([0, 2050, total], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    _run(ctx, torch, kern, "hi")
    rows = np.r_[0:3, 2046:2200]
    got = _host(big[:, 3:4].contiguous())
    del big, kern
    qd, kd, vd = (obf16.decode(t) for t in (q, k, v))
    for a, b in ((0, 3), (2050, total)):
        want, mass = OS.attn_prompt(qd, kd, vd, [0 if a == 0 else 2050, b])
        _attn_ok(got[a:b], want[a:b], mass[a:b])
    want, mass = OS._attend(qd[2049, 0], kd[:2050, 0], vd[:2050, 0], dim ** -0.5)
    _attn_ok(got[2049, 0], want, mass)
    assert rows.size


def test_prompt_workers_pause_inside_a_block_and_go_on(env):
    """A pausing request while a long prompt runs as workers: the job stops or pauses, goes on, and gives the
    original form's bits."""
    B, ctx, torch = env
    total = 12000
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn((total, 8, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    cu = torch.tensor([0, total], dtype=torch.int32, device="cuda")
    a, b = torch.zeros_like(q), torch.zeros_like(q)
    torch.cuda.synchronize()
    ctx.launch_native(B.attn_prompt_bf16(q, k, v, a, cu))
    torch.cuda.synchronize()
    kern = B.attn_prompt_bf16(q, k, v, b, cu)
    job = ctx.launch_ptb(kern, 256, coverage=True)
    stops = 0
    for _ in range(200):
        job.preempt(pause=True)
        job.end_pause()
        if job.wait() == B.JOB_COMPLETE:
            break
        stops += 1
        job.resume()
    assert job.wait() == B.JOB_COMPLETE
    assert (job.coverage()["count"] == 1).all()
    job.free()
    torch.cuda.synchronize()
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("dim,every,chunk", [(128, 4, 1), (64, 1, 1), (128, 16, 4), (64, 64, 2)])
def test_prompt_workers_that_are_asked_to_pause_wait_inside_their_blocks(env, dim, every, chunk):
    """A request that is held for 4 ms, several times a block's time and more than the whole kernel's, keeps the workers where
    they are (they would have left otherwise); withdrawn, they finish their blocks and leave, and go on when resumed.  The bits
    are those of the original form, with every block executed once."""
    import time
    B, ctx, torch = env
    total = 16384
    g = torch.Generator(device="cuda").manual_seed(dim + every)
    q, k, v = (torch.randn((total, 16, dim), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    cu = torch.tensor([0, total], dtype=torch.int32, device="cuda")
    want, out = torch.zeros_like(q), torch.zeros_like(q)
    torch.cuda.synchronize()
    ctx.launch_native(B.attn_prompt_bf16(q, k, v, want, cu))
    torch.cuda.synchronize()
    kern = B.attn_prompt_bf16(q, k, v, out, cu)
    ctx.set_yield_bound_us(100000)
    ctx.set_yield_every(every)
    try:
        spans = []
        for pauses in (0, 0, 2):
            out.zero_()
            torch.cuda.synchronize()
            t0 = time.perf_counter()
            job = ctx.launch_ptb(kern, 256, chunk=chunk, coverage=True)
            stops = 0
            for _ in range(pauses):
                while time.perf_counter() < t0 + 0.2 * spans[-1]:
                    pass
                job.preempt(pause=True)
                time.sleep(0.004)
                job.pump()
                assert job.progress()[2] == B.JOB_RUNNING
                job.end_pause()
                if job.wait() == B.JOB_STOPPED:
                    stops += 1
                    t0 = time.perf_counter()
                    job.resume()
            assert job.wait() == B.JOB_COMPLETE
            if pauses:
                assert stops >= 1
            else:
                spans.append(time.perf_counter() - t0)
            assert (job.coverage()["count"] == 1).all()
            job.free()
            torch.cuda.synchronize()
            assert torch.equal(out.view(torch.int16), want.view(torch.int16))
        assert 0.0003 < spans[-1] < 0.003                  # (otherwise the pauses prove nothing)
    finally:
        ctx.set_yield_bound_us(1000)
        ctx.set_yield_every(4)


def test_prompt_blocks_too_short_to_pause_inside_pause_before_the_next_of_their_fetch(env):
    """Blocks of two and four tiles with looks 16 tiles apart: of the 64 blocks of a fetch the next one waits."""
    import time
    B, ctx, torch = env
    seqs, total = 800, 160000
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k, v = (torch.randn((total, 2, 64), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    cu = torch.arange(seqs + 1, dtype=torch.int32, device="cuda") * 200
    want, out = torch.zeros_like(q), torch.zeros_like(q)
    torch.cuda.synchronize()
    ctx.launch_native(B.attn_prompt_bf16(q, k, v, want, cu))
    torch.cuda.synchronize()
    kern = B.attn_prompt_bf16(q, k, v, out, cu)
    ctx.set_yield_bound_us(100000)
    ctx.set_yield_every(16)
    try:
        job = ctx.launch_ptb(kern, 2, chunk=64, coverage=True)
        time.sleep(0.0005)
        job.preempt(pause=True)
        time.sleep(0.01)
        job.pump()
        assert job.progress()[2] == B.JOB_RUNNING
        job.end_pause()
        assert job.wait() == B.JOB_STOPPED and 0 < job.progress()[0] < kern.total_blocks
        job.resume()
        assert job.wait() == B.JOB_COMPLETE
        assert (job.coverage()["count"] == 1).all()
        job.free()
    finally:
        ctx.set_yield_bound_us(1000)
        ctx.set_yield_every(4)
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), want.view(torch.int16))


# ---------------------------------------------------------------- behind a shared prefix
def _prefix(seed, batch, heads, kv, dim, prefix, cap):
    rng = np.random.default_rng(seed)
    return (_bits(rng, (batch, heads, dim)), _bits(rng, (prefix, kv, dim)), _bits(rng, (prefix, kv, dim)),
            _bits(rng, (batch, cap, kv, dim)), _bits(rng, (batch, cap, kv, dim)))


def _scratch(B, torch, batch, heads, kv, dim, prefix, cap):
    n = B.attn_prefix_scratch_bytes(batch, heads, kv, dim, prefix, cap)
    return torch.full((max(n, 1) + 64,), 0x7F, dtype=torch.uint8, device="cuda")   # (as floats: NaN-like garbage)


PREFIX = [
    # batch, heads, kv_heads, dim, prefix, own_cap, lens
    (1, 1, 1, 128, 1, 0, None), (1, 1, 1, 64, 0, 1, [1]), (2, 2, 1, 128, 31, 5, [0, 5]), (3, 4, 2, 64, 32, 33, [33, 0, 1]),
    (3, 4, 2, 128, 33, 64, [64, 63, 32]), (5, 7, 1, 128, 127, 65, [65, 0, 31, 33, 64]), (4, 12, 12, 64, 300, 20, [3, 0, 20, 7]),
    # nothing to attend to, lengths outside the cache
    (3, 2, 2, 128, 0, 40, [0, 40, -3]), (3, 2, 1, 64, 10, 8, [99, -1, 8]), (2, 2, 2, 64, 0, 0, None),
    # more than 64 rows to a K/V head, several workgroups' worth of them, more than 64 heads to one
    (40, 4, 2, 128, 200, 9, "even"), (70, 8, 4, 64, 129, 3, "even"), (300, 1, 1, 128, 64, 2, "even"), (3, 96, 1, 128, 70, 90, [90, 0, 45]),
    (2, 140, 2, 64, 65, 66, [66, 1]), (1, 70, 1, 128, 40, 0, None),
    # everything of a sequence in one workgroup: a prefix that ends inside a tile and as many as a wave has, long ones of many sequences
    (3, 8, 4, 128, 200, 300, [300, 0, 77]), (2, 16, 1, 128, 128, 128, [128, 1]), (4, 6, 2, 64, 97, 900, [900, 0, 1, 31]),
    (128, 4, 2, 64, 0, 1100, "even"), (130, 2, 2, 128, 7, 600, "even"),
    # in parts: 16 rows of the prefix, more than 16, more than 64
    (1, 16, 1, 128, 4000, 0, None), (2, 16, 2, 64, 2500, 1300, [1300, 1299]), (6, 8, 2, 64, 1500, 100, "even"), (20, 8, 2, 128, 700, 600, "even"),
    # many rows and a long prefix (128-row workgroups): several of them, one of few rows, more than 16 heads to a K/V head
    (40, 16, 1, 64, 13200, 40, "even"), (33, 10, 2, 128, 25500, 70, "even"), (3, 96, 1, 128, 29200, 90, [90, 0, 45]),
]


@pytest.mark.parametrize("batch,heads,kv,dim,prefix,cap,lens", PREFIX)
@pytest.mark.parametrize("hi", [True, False])
def test_prefix_attention(env, batch, heads, kv, dim, prefix, cap, lens, hi):
    B, ctx, torch = env
    q, K, V, Ko, Vo = _prefix(batch + prefix, batch, heads, kv, dim, prefix, cap)
    lens = [i % (cap + 1) for i in range(batch)] if lens == "even" else lens or [0] * batch
    hidden = [min(max(n, 0), cap) for n in lens]
    Kn, Vn = Ko.copy(), Vo.copy()
    for b, n in enumerate(hidden):                         # what lies behind is no numbers
        Kn[b, n:], Vn[b, n:] = 0x7FC0, 0xFF80
    out = torch.full((batch, heads, dim), SENTINEL, dtype=torch.int16, device="cuda")
    kern = B.attn_prefix_bf16(_dev(torch, q), _dev(torch, K), _dev(torch, V), _dev(torch, Kn), _dev(torch, Vn),
                              torch.tensor(lens, dtype=torch.int32, device="cuda"), out, _scratch(B, torch, batch, heads, kv, dim, prefix, cap))
    torch.cuda.synchronize()
    _run(ctx, torch, kern, "hi" if hi else "be")
    want, mass = OS.attn_prefix(*(obf16.decode(t) for t in (q, K, V, Ko, Vo)), lens)
    got = _host(out)
    _attn_ok(got, want, mass)
    for b, n in enumerate(hidden):
        if prefix + n == 0:
            assert (got[b] == 0).all()


def test_prefix_many_parts(env):
    """A prefix and replies that are split into many parts, some of them beyond a reply's end."""
    B, ctx, torch = env
    batch, heads, kv, dim, prefix, cap = 2, 2, 1, 128, 20000, 9000
    q, K, V, Ko, Vo = _prefix(5, batch, heads, kv, dim, prefix, cap)
    lens = [9000, 130]
    out = torch.zeros((batch, heads, dim), dtype=torch.int16, device="cuda")
    kern = B.attn_prefix_bf16(_dev(torch, q), _dev(torch, K), _dev(torch, V), _dev(torch, Ko), _dev(torch, Vo),
                              torch.tensor(lens, dtype=torch.int32, device="cuda"), out, _scratch(B, torch, batch, heads, kv, dim, prefix, cap))
    torch.cuda.synchronize()
    _run(ctx, torch, kern, "hi")
    want, mass = OS.attn_prefix(*(obf16.decode(t) for t in (q, K, V, Ko, Vo)), lens)
    _attn_ok(_host(out), want, mass)


def test_prefix_strides_and_caches_beyond_32_bits(env):
    """Padded tokens everywhere, and sequences' caches 2^31 elements apart."""
    B, ctx, torch = env
    batch, heads, kv, dim, prefix, cap = 2, 4, 2, 64, 50, 40
    q, K, V, Ko, Vo = _prefix(6, batch, heads, kv, dim, prefix, cap)
    lens = [40, 17]
    both = _dev(torch, np.concatenate([K, V], 1))          # [prefix, 2 kv, dim]
    big = torch.empty((1 << 31) + cap * 2 * kv * dim, dtype=torch.int16, device="cuda")
    own = big.as_strided((batch, cap, 2 * kv, dim), (1 << 31, 2 * kv * dim, dim, 1))
    own.copy_(_dev(torch, np.concatenate([Ko, Vo], 2)))
    qq = torch.zeros((batch, heads + 2, dim), dtype=torch.int16, device="cuda")
    qq[:, 1:1 + heads] = _dev(torch, q)
    out = torch.full((batch, heads + 1, dim), SENTINEL, dtype=torch.int16, device="cuda")
    kern = B.attn_prefix_bf16(qq[:, 1:1 + heads], both[:, :kv], both[:, kv:], own[:, :, :kv], own[:, :, kv:],
                              torch.tensor(lens, dtype=torch.int32, device="cuda"), out[:, :heads],
                              _scratch(B, torch, batch, heads, kv, dim, prefix, cap), scale=0.2)
    torch.cuda.synchronize()
    _run(ctx, torch, kern, "hi")
    got = _host(out)
    del big, own, kern
    want, mass = OS.attn_prefix(*(obf16.decode(t) for t in (q, K, V, Ko, Vo)), lens, 0.2)
    _attn_ok(got[:, :heads], want, mass)
    assert (got[:, heads:] == SENTINEL).all()


# batch, heads, kv_heads, dim, prefix, own_cap: all of a sequence in a workgroup, and in parts of 16, 64 and 128 rows of the prefix
WAYS = [(3, 4, 2, 64, 150, 200), (2, 16, 2, 128, 2200, 700), (3, 16, 2, 64, 2200, 700), (40, 96, 6, 128, 2200, 40)]


@pytest.mark.parametrize("batch,heads,kv,dim,prefix,cap", WAYS)
def test_prefix_large_scores(env, batch, heads, kv, dim, prefix, cap):
    """A maximum that keeps rising, in the prefix and beyond it in a sequence's own tokens, to about e^10 times the
    first weights.  (sum |q k| stays below 13: scores are off by 130 x 13 x 2^-24 < 2^-13.2, and numerator and
    denominator by as much of M each, below 2^-12 together.)"""
    B, ctx, torch = env
    rng = np.random.default_rng(batch)
    base = rng.standard_normal(dim)
    base *= (dim / (base @ base)) ** 0.5
    near = lambda shape, times: TI.to_bf16_bits((times * base + 0.3 * rng.standard_normal(shape)).astype(np.float32))
    ramp = lambda n, lo, hi: np.linspace(lo, hi, n)[:, None, None]
    q, K, Ko = near((batch, heads, dim), 1.0), near((prefix, kv, dim), ramp(prefix, 0.1, 1.0)), near((batch, cap, kv, dim), ramp(cap, 1.0, 1.6))
    V, Vo = _bits(rng, (prefix, kv, dim)), _bits(rng, (batch, cap, kv, dim))
    lens = [cap - 3 * b if b % 4 else 0 for b in range(batch)]
    scale = 6.0 / dim
    out = torch.zeros((batch, heads, dim), dtype=torch.int16, device="cuda")
    kern = B.attn_prefix_bf16(*(_dev(torch, t) for t in (q, K, V, Ko, Vo)), torch.tensor([max(n, 0) for n in lens], dtype=torch.int32, device="cuda"),
                              out, _scratch(B, torch, batch, heads, kv, dim, prefix, cap), scale=scale)
    torch.cuda.synchronize()
    _run(ctx, torch, kern, "hi")
    want, mass = OS.attn_prefix(*(obf16.decode(t) for t in (q, K, V, Ko, Vo)), lens, scale)
    _attn_ok(_host(out), want, mass)


@pytest.mark.parametrize("batch,heads,kv,dim,prefix,cap", WAYS[1:])
def test_prefix_tokens_as_far_apart_as_they_may_be(env, batch, heads, kv, dim, prefix, cap):
    """2^20 elements between the prefix's tokens: more than 2^32 bytes in all, in each way of cutting a call up."""
    B, ctx, torch = env
    q, K, V, Ko, Vo = _prefix(batch + dim, batch, heads, kv, dim, prefix, cap)
    lens = [(7 * b) % (cap + 1) for b in range(batch)]
    far = torch.empty((prefix, 1 << 20), dtype=torch.int16, device="cuda")
    K1, V1 = (far[:, at:at + kv * dim].unflatten(1, (kv, dim)) for at in (0, kv * dim))
    K1.copy_(_dev(torch, K))
    V1.copy_(_dev(torch, V))
    out = torch.zeros((batch, heads, dim), dtype=torch.int16, device="cuda")
    kern = B.attn_prefix_bf16(_dev(torch, q), K1, V1, _dev(torch, Ko), _dev(torch, Vo), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                              out, _scratch(B, torch, batch, heads, kv, dim, prefix, cap))
    torch.cuda.synchronize()
    _run(ctx, torch, kern, "hi")
    got = _host(out)
    del far, K1, V1, kern
    want, mass = OS.attn_prefix(*(obf16.decode(t) for t in (q, K, V, Ko, Vo)), lens)
    _attn_ok(got, want, mass)


@pytest.mark.parametrize("batch,heads,kv,dim,prefix,cap", WAYS)
def test_prefix_captured_twice_with_scratch_of_its_own(env, batch, heads, kv, dim, prefix, cap):
    """Two graphs of the same call, replayed in turn and with eager calls between them; lengths change in place."""
    B, ctx, torch = env
    g = torch.Generator(device="cuda").manual_seed(6)
    t = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    q, K, V, Ko, Vo = t(batch, heads, dim), t(prefix, kv, dim), t(prefix, kv, dim), t(batch, cap, kv, dim), t(batch, cap, kv, dim)
    lens = torch.full((batch,), cap, dtype=torch.int32, device="cuda")
    outs = [torch.zeros_like(q) for _ in range(3)]
    calls = [B.attn_prefix_bf16(q, K, V, Ko, Vo, lens, o, _scratch(B, torch, batch, heads, kv, dim, prefix, cap)) for o in outs]
    torch.cuda.synchronize()
    graphs = []
    for kern in calls[:2]:
        ctx.launch_native(kern, hi=True)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=ctx._streams[0]):
            ctx.launch_native(kern, hi=True)
    for turn in range(4):
        lens.copy_((torch.arange(batch, device="cuda") * (5 + turn) + turn) % (cap + 1))
        q.copy_(torch.randn(q.shape, generator=g, device="cuda"))
        torch.cuda.synchronize()
        graphs[0].replay()
        torch.cuda.synchronize()
        ctx.launch_native(calls[2], hi=True)
        torch.cuda.synchronize()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o.view(torch.int16), outs[2].view(torch.int16)) for o in outs[:2]), turn
        assert outs[2].float().abs().sum() > 0


@pytest.mark.parametrize("poison", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("low", ["prefix", "own"])
@pytest.mark.parametrize("batch,heads,kv,dim,prefix,cap", WAYS)
def test_prefix_what_a_token_holds_is_seen_whatever_its_weight(env, batch, heads, kv, dim, prefix, cap, low, poison):
    """V of one token is no number, in a stretch of tokens (the first half of the prefix, or a sequence's own) whose
    scores lie 300 below the others': its weight is zero in 32 bits, and zero times it is not zero.
    (Scores of magnitude S are off by (dim + 2) S 2^-24, and p by as much of itself, in numerator and denominator.)"""
    B, ctx, torch = env
    rng = np.random.default_rng(batch + dim)
    base = rng.standard_normal(dim)
    base *= (dim / (base @ base)) ** 0.5
    near = lambda shape, times: (times * base + 0.1 * rng.standard_normal(shape)).astype(np.float32)
    q, K, Ko = near((batch, heads, dim), 1.0), near((prefix, kv, dim), 1.0), near((batch, cap, kv, dim), 1.0)
    V, Vo = _bits(rng, (prefix, kv, dim)), _bits(rng, (batch, cap, kv, dim))
    lens = [cap - b % 4 for b in range(batch)]
    hit = rng.integers(0, prefix // 2), rng.integers(0, min(lens))
    bad = TI.to_bf16_bits(np.float32([poison]))[0]
    clean = V.copy(), Vo.copy()
    if low == "prefix":
        K[:prefix // 2] *= -1
        V[hit[0], kv - 1, 5:9] = bad
    else:
        Ko *= -1
        Vo[batch - 1, hit[1], kv - 1, 5:9] = bad
    q, K, Ko = (TI.to_bf16_bits(t) for t in (q, K, Ko))
    scale = 150.0 / dim
    out = torch.zeros((batch, heads, dim), dtype=torch.int16, device="cuda")
    kern = B.attn_prefix_bf16(*(_dev(torch, t) for t in (q, K, V, Ko, Vo)), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                              out, _scratch(B, torch, batch, heads, kv, dim, prefix, cap), scale=scale)
    torch.cuda.synchronize()
    _run(ctx, torch, kern, "hi")
    qd, Kd, Kod = (obf16.decode(t) for t in (q, K, Ko))
    want, mass = OS.attn_prefix(qd, Kd, obf16.decode(clean[0]), Kod, obf16.decode(clean[1]), lens, scale)
    hits = np.zeros(want.shape, bool)
    hits[0 if low == "prefix" else batch - 1:, heads - heads // kv:, 5:9] = True
    got = obf16.decode(_host(out))
    assert not np.isfinite(got[hits]).any()
    S = scale * np.sqrt((qd ** 2).sum(-1).max() * max((Kd ** 2).sum(-1).max(), (Kod ** 2).sum(-1).max()))
    bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -12 + 2 * (dim + 2) * S * 2.0 ** -24) * mass
    assert (np.abs(got - want) <= bound)[~hits].all()


@pytest.mark.parametrize("batch,heads,kv,dim,prefix,cap", WAYS + [(2, 16, 2, 128, 0, 3000), (2, 4, 2, 64, 0, 60)])
def test_prefix_without_a_token_gives_zeros_and_without_a_finite_score_none(env, batch, heads, kv, dim, prefix, cap):
    """Scores of -inf throughout have no softmax: NaN, as in a prompt.  Zeros stand where there is no token."""
    B, ctx, torch = env
    q, K, V, Ko, Vo = _prefix(batch, batch, heads, kv, dim, prefix, cap)
    q = q & np.uint16(0x7FFF) | np.uint16(0x3C00)          # (positive, so that no product is +inf)
    K[:], Ko[:] = 0xFF80, 0xFF80
    lens = [0 if b % 2 else cap for b in range(batch)]
    out = torch.full((batch, heads, dim), SENTINEL, dtype=torch.int16, device="cuda")
    kern = B.attn_prefix_bf16(*(_dev(torch, t) for t in (q, K, V, Ko, Vo)), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                              out, _scratch(B, torch, batch, heads, kv, dim, prefix, cap))
    torch.cuda.synchronize()
    _run(ctx, torch, kern, "hi")
    got = obf16.decode(_host(out))
    for b, n in enumerate(lens):
        assert np.isnan(got[b]).all() if prefix + n else (got[b] == 0).all(), b


@pytest.mark.parametrize("batch,heads,kv,dim,prefix,cap,lens", [(1, 7, 1, 128, 4000, 64, [64]), (1, 1, 1, 64, 4480, 0, [0]),
                                                                (1, 35, 5, 64, 1100, 700, [699])])
def test_prefix_with_an_odd_number_of_partial_results(env, batch, heads, kv, dim, prefix, cap, lens):
    """The weighted sums in scratch begin at a multiple of 16 bytes, and end where the scratch does."""
    B, ctx, torch = env
    q, K, V, Ko, Vo = _prefix(heads + prefix, batch, heads, kv, dim, prefix, cap)
    n = B.attn_prefix_scratch_bytes(batch, heads, kv, dim, prefix, cap)
    assert n % 16 == 0 and (n // (dim * 4 + 8)) % 2 == 1   # (an odd number of records of dim floats and two)
    room = torch.full((n + 64,), 0x7F, dtype=torch.uint8, device="cuda")
    out = torch.zeros((batch, heads, dim), dtype=torch.int16, device="cuda")
    kern = B.attn_prefix_bf16(*(_dev(torch, t) for t in (q, K, V, Ko, Vo)), torch.tensor(lens, dtype=torch.int32, device="cuda"), out, room)
    torch.cuda.synchronize()
    _run(ctx, torch, kern, "hi")
    want, mass = OS.attn_prefix(*(obf16.decode(t) for t in (q, K, V, Ko, Vo)), lens)
    _attn_ok(_host(out), want, mass)
    assert (room[n:] == 0x7F).all()


@pytest.mark.parametrize("dim", [64, 128])
def test_attention_takes_scores_of_2_24_and_values_of_2_96(env, dim):
    """Scores of 2^17, 2 x 2^17 ... 2^24, each the largest so far: its token's weight is one, all others' zero, and the output
    is its V, to the bit (a product with p and a division by the same p, off by 2^-23 in all before the last rounding)."""
    B, ctx, torch = env
    n = 128
    rng = np.random.default_rng(dim)
    k = np.zeros((n, 1, dim), np.float32)
    k[:, 0, 5] = (1 + np.arange(n)) * 2.0 ** 17            # (8 bits each)
    q = np.zeros((n, 2, dim), np.float32)
    q[:, :, 5] = 1.0
    v = TI.to_bf16_bits((np.sign(rng.standard_normal((n, 1, dim))) * 2.0 ** rng.uniform(90, 96, (n, 1, dim))).astype(np.float32))
    q, k = TI.to_bf16_bits(q), TI.to_bf16_bits(k)
    out = torch.zeros((n, 2, dim), dtype=torch.int16, device="cuda")
    qd, kd, vd = (_dev(torch, t) for t in (q, k, v))
    prompt = B.attn_prompt_bf16(qd, kd, vd, out, torch.tensor([0, n], dtype=torch.int32, device="cuda"), scale=1.0)
    torch.cuda.synchronize()
    _run(ctx, torch, prompt, "hi")
    assert (_host(out) == v).all()
    for prefix, cap in ((n, 0), (0, n), (50, n - 50)):
        lens = torch.tensor([cap, 0][:2 if prefix else 1], dtype=torch.int32, device="cuda")
        batch = lens.numel()
        one = torch.zeros((batch, 2, dim), dtype=torch.int16, device="cuda")
        own = [t[prefix:].unsqueeze(0).repeat(batch, 1, 1, 1) for t in (kd, vd)]
        step = B.attn_prefix_bf16(qd[:batch], kd[:prefix], vd[:prefix], *own, lens, one, _scratch(B, torch, batch, 2, 1, dim, prefix, cap), scale=1.0)
        torch.cuda.synchronize()
        _run(ctx, torch, step, "hi")
        got = _host(one)
        assert (got[0] == v[-1]).all() and (batch == 1 or (got[1] == v[prefix - 1]).all())


def test_prefix_is_not_transformable(env):
    B, ctx, torch = env
    z = torch.zeros((1, 1, 64), dtype=torch.int16, device="cuda")
    kern = B.attn_prefix_bf16(z, z, z, None, None, None, z.clone(), torch.zeros(4096, dtype=torch.uint8, device="cuda"))
    for launch in (lambda: ctx.launch_ptb(kern, 1), lambda: ctx.launch_sliced(kern, 1)):
        with pytest.raises(B.TallyError) as e:
            launch()
        assert e.value.status == B.ERR_UNSUPPORTED


# ---------------------------------------------------------------- 4-bit products
def _w4(rng, m, n, k, group, zeros):
    groups = -(-k // group)
    return (_bits(rng, (m, k)), rng.integers(0, 16, (n, k)), TI.to_bf16_bits(rng.uniform(0.5, 2.0, (n, groups)).astype(np.float32)),
            rng.integers(0, 16, (n, groups)).astype(np.uint8) if zeros else None)


def _w4_ok(got_bits, x, codes, scales, zeros, group):
    want, mass = OS.gemv_w4(obf16.decode(x), codes, obf16.decode(scales), zeros, group)
    err = np.abs(obf16.decode(got_bits) - want)
    bound = 2.0 ** -8 * np.abs(want) + (2 * x.shape[1] + 300) * 2.0 ** -24 * mass
    assert (err <= bound).all(), f"worst {(err / bound).max():.2f} bounds"


W4 = [(1, 1, 8, 32, False), (1, 16, 128, 128, True), (2, 17, 120, 32, True), (3, 15, 136, 64, False), (16, 33, 1000, 32, True),
      (5, 100, 512, 64, True), (4, 50, 640, 256, False), (16, 64, 1288, 128, True), (7, 31, 2056, 64, False), (1, 300, 4096, 128, False),
      (9, 48, 4104, 384, True), (16, 16, 72, 64, True), (1, 40, 11008, 64, True),
      # vectors that just fit into LDS, and that just do not
      (1, 33, 11264, 128, False), (1, 33, 11272, 32, True), (1, 20, 11776, 64, False), (1, 16, 12000, 128, True)]


@pytest.mark.parametrize("form", ["hi", "be", "sliced", "ptb"])
@pytest.mark.parametrize("m,n,k,group,zeros", W4)
def test_gemv_w4(env, m, n, k, group, zeros, form):
    B, ctx, torch = env
    rng = np.random.default_rng(n + k)
    x, codes, scales, z = _w4(rng, m, n, k, group, zeros)
    W = B.pack_w4(torch.from_numpy(codes))
    s, zp = B.pack_w4_groups(torch.from_numpy(scales.view(np.int16))), B.pack_w4_groups(torch.from_numpy(z)) if zeros else None
    # rows and columns that do not exist hold garbage
    junk = torch.from_numpy(rng.integers(0, 16, (W.shape[0] * 16, W.shape[1] * 128)))
    junk[:n, :k] = torch.from_numpy(codes)
    W = B.pack_w4(junk)
    if n % 16:
        s[-1, :, n % 16:] = 0x7FC0
    y = torch.full((m, n), SENTINEL, dtype=torch.int16, device="cuda")
    kern = B.gemv_w4_bf16(_dev(torch, x), W.cuda(), s.cuda(), y, zeros=zp.cuda() if zeros else None, group=group)
    torch.cuda.synchronize()
    _run(ctx, torch, kern, form)
    _w4_ok(_host(y), x, codes, scales, z, group)


def test_gemv_w4_strides_and_neighbours(env):
    """Vectors and outputs with padded rows; what lies between and behind them is left alone, and not read
    into sums even if it is no number."""
    B, ctx, torch = env
    m, n, k, group = 3, 37, 200, 32
    rng = np.random.default_rng(11)
    x, codes, scales, z = _w4(rng, m, n, k, group, True)
    wide = np.full((m + 1, k + 24), 0x7FC0, np.uint16)
    wide[:m, :k] = x
    xd = _dev(torch, wide)
    y = torch.full((m + 2, n + 5), SENTINEL, dtype=torch.int16, device="cuda")
    kern = B.gemv_w4_bf16(xd[:m, :k], B.pack_w4(torch.from_numpy(codes)).cuda(), B.pack_w4_groups(torch.from_numpy(scales.view(np.int16))).cuda(),
                          y[1:1 + m, 2:2 + n], zeros=B.pack_w4_groups(torch.from_numpy(z)).cuda(), group=group)
    torch.cuda.synchronize()
    _run(ctx, torch, kern, "hi")
    got = _host(y)
    _w4_ok(got[1:1 + m, 2:2 + n], x, codes, scales, z, group)
    assert (got[0] == SENTINEL).all() and (got[1 + m:] == SENTINEL).all()
    assert (got[1:1 + m, :2] == SENTINEL).all() and (got[1:1 + m, 2 + n:] == SENTINEL).all()


@pytest.mark.parametrize("m,k,group", [(1, 8200, 128), (3, 520, 32), (16, 1000, 64), (5, 640, 256)])
def test_gemv_w4_takes_vectors_of_2_112(env, m, k, group):
    """x as large as the header allows, scales as small: nothing overflows on the way."""
    B, ctx, torch = env
    n = 50
    x, codes, scales, z = _w4(np.random.default_rng(k), m, n, k, group, True)
    x = TI.to_bf16_bits((np.clip(obf16.decode(x), -3.9, 3.9) * 2.0 ** 110).astype(np.float32))
    scales = TI.to_bf16_bits((obf16.decode(scales) * 2.0 ** -112).astype(np.float32))
    y = torch.zeros((m, n), dtype=torch.int16, device="cuda")
    kern = B.gemv_w4_bf16(_dev(torch, x), B.pack_w4(torch.from_numpy(codes)).cuda(), B.pack_w4_groups(torch.from_numpy(scales.view(np.int16))).cuda(),
                          y, zeros=B.pack_w4_groups(torch.from_numpy(z)).cuda(), group=group)
    torch.cuda.synchronize()
    _run(ctx, torch, kern, "hi")
    _w4_ok(_host(y), x, codes, scales, z, group)


def test_gemv_w4_rows_do_not_depend_on_the_number_of_vectors(env):
    B, ctx, torch = env
    n, k, group = 100, 1000, 64
    x, codes, scales, z = _w4(np.random.default_rng(12), 16, n, k, group, False)
    W, s, xd = B.pack_w4(torch.from_numpy(codes)).cuda(), B.pack_w4_groups(torch.from_numpy(scales.view(np.int16))).cuda(), _dev(torch, x)
    outs = []
    for m in (1, 2, 5, 16):
        y = torch.zeros((m, n), dtype=torch.int16, device="cuda")
        kern = B.gemv_w4_bf16(xd[:m], W, s, y, group=group)
        torch.cuda.synchronize()
        _run(ctx, torch, kern, "hi")
        outs.append(_host(y))
    assert all((o == outs[-1][:len(o)]).all() for o in outs)


# m, n, rows of tiles of a workgroup, k, group, zeros: every kernel with more than one row, the last workgroup with all of
# its rows and without one, two or three of them, its last row with all of its 16 rows of weights and without some
W4_ROWS = [
    (1, 16401, 2, 72, 32, True), (2, 16400, 2, 296, 64, False), (1, 16390, 2, 264, 128, True), (4, 4117, 2, 1160, 128, False),
    (3, 4100, 2, 136, 64, True), (6, 4112, 2, 2200, 32, False),
    (8, 8213, 3, 1288, 32, True), (16, 8230, 3, 200, 64, False), (10, 8208, 3, 296, 128, True), (7, 8240, 3, 1160, 256, False), (8, 16405, 3, 128, 64, True),
    (16, 24600, 4, 72, 64, True), (13, 24580, 4, 264, 32, False), (16, 24624, 4, 1160, 128, True), (11, 24640, 4, 136, 384, False),
]


@pytest.mark.parametrize("m,n,rows,k,group,zeros", W4_ROWS)
def test_gemv_w4_with_several_rows_of_tiles(env, m, n, rows, k, group, zeros):
    """In every form; what stands for rows and columns that do not exist is garbage, and y's neighbours stay."""
    B, ctx, torch = env
    rng = np.random.default_rng(n + k)
    x, codes, scales, z = _w4(rng, m, n, k, group, zeros)
    junk = torch.from_numpy(rng.integers(0, 16, (-(-n // 16) * 16, -(-k // 128) * 128)))
    junk[:n, :k] = torch.from_numpy(codes)
    W, s = B.pack_w4(junk).cuda(), B.pack_w4_groups(torch.from_numpy(scales.view(np.int16)))
    if n % 16:
        s[-1, :, n % 16:] = 0x7FC0
    zp = B.pack_w4_groups(torch.from_numpy(z)).cuda() if zeros else None
    xd, s = _dev(torch, x), s.cuda()
    want, mass = OS.gemv_w4(obf16.decode(x), codes, obf16.decode(scales), z, group)
    bound = 2.0 ** -8 * np.abs(want) + (2 * k + 300) * 2.0 ** -24 * mass
    outs = []
    for form in ("hi", "be", "sliced", "ptb"):
        y = torch.full((m + 1, n), SENTINEL, dtype=torch.int16, device="cuda")
        kern = B.gemv_w4_bf16(xd, W, s, y[:m], zeros=zp, group=group)
        assert kern.grid == (-(-n // (16 * rows)), 1, 1)
        torch.cuda.synchronize()
        _run(ctx, torch, kern, form)
        outs.append(_host(y))
        err = np.abs(obf16.decode(outs[-1][:m]) - want)
        assert (err <= bound).all(), f"{form}: worst {(err / bound).max():.2f} bounds"
        assert (outs[-1][m] == SENTINEL).all(), form
    assert all((o == outs[0]).all() for o in outs)


@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True), (384, False)])
@pytest.mark.parametrize("n,k,kernels", [(24596, 520, {(1, 2), (4, 2), (8, 3), (16, 4)}), (8210, 1000, {(1, 1), (3, 1), (4, 2), (10, 3)}),
                                         (16410, 9000, {(1, 2), (4, 2), (16, 3)})])
def test_gemv_w4_bits_do_not_depend_on_the_kernel(env, n, k, kernels, group, zeros):
    """Every row's bits are the same with one to sixteen vectors, one to four rows of tiles, and (one vector, k = 9000, few
    rows) with x in LDS."""
    B, ctx, torch = env
    g = torch.Generator(device="cuda").manual_seed(n)
    tiles, groups = -(-n // 16), -(-k // group)
    W = torch.randint(-(1 << 31), 1 << 31, (tiles, -(-k // 128), 64, 4), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    s = torch.rand((tiles, groups, 16), generator=g, device="cuda").to(torch.bfloat16)
    zp = torch.randint(0, 17, (tiles, groups, 16), generator=g, device="cuda", dtype=torch.uint8) if zeros else None
    x = torch.randn((16, k), generator=g, device="cuda").to(torch.bfloat16)
    outs = []
    for m, rows in sorted(kernels):
        y = torch.zeros((m, n), dtype=torch.bfloat16, device="cuda")
        kern = B.gemv_w4_bf16(x[:m], W, s, y, zeros=zp, group=group)
        assert kern.grid[0] == -(-tiles // rows)
        torch.cuda.synchronize()
        ctx.launch_native(kern, hi=True)
        outs.append(y)
    for rows in (16, 100, 4096):                           # (one row of tiles each; with one vector of 9000, x is in LDS)
        y = torch.zeros((1, rows), dtype=torch.bfloat16, device="cuda")
        part = -(-rows // 16)
        kern = B.gemv_w4_bf16(x[:1], W[:part], s[:part], y, zeros=zp[:part] if zeros else None, group=group)
        assert kern.grid[0] == part
        torch.cuda.synchronize()
        ctx.launch_native(kern, hi=True)
        outs.append(y)
    torch.cuda.synchronize()
    whole = outs[len(kernels) - 1].view(torch.int16)
    assert whole.shape[0] >= 10 and torch.isfinite(outs[len(kernels) - 1].float()).all()
    for o in outs:
        assert torch.equal(o.view(torch.int16), whole[:o.shape[0], :o.shape[1]]), o.shape


# ---------------------------------------------------------------- as a program uses them
def _decode_step(B, torch, g, batch, heads, kv, dim, prefix_kv, cap):
    """A batch's decode step behind a prefix: attention, then two 4-bit products of its output."""
    hidden = heads * dim
    t = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    q, own = t(batch, heads, dim), t(batch, cap, 2 * kv, dim)
    lens = torch.arange(batch, dtype=torch.int32, device="cuda") * cap // max(batch - 1, 1)
    out, mid, y = torch.zeros_like(q), torch.zeros((batch, 512), dtype=torch.bfloat16, device="cuda"), torch.zeros((batch, hidden), dtype=torch.bfloat16, device="cuda")
    prefix = prefix_kv.shape[0]
    room = torch.empty(B.attn_prefix_scratch_bytes(batch, heads, kv, dim, prefix, cap), dtype=torch.uint8, device="cuda")
    def w(n, k):
        return (B.pack_w4(torch.randint(0, 16, (n, k), generator=g, device="cuda")),
                B.pack_w4_groups((torch.rand((n, k // 128), generator=g, device="cuda") / k ** 0.5).to(torch.bfloat16)))
    (w1, s1), (w2, s2) = w(512, hidden), w(hidden, 512)
    kernels = [B.attn_prefix_bf16(q, prefix_kv[:, :kv], prefix_kv[:, kv:], own[:, :, :kv], own[:, :, kv:], lens, out, room),
               B.gemv_w4_bf16(out.view(batch, hidden), w1, s1, mid), B.gemv_w4_bf16(mid, w2, s2, y)]
    return kernels, (out, mid, y)


def test_decode_requests_beside_prompts_under_the_scheduler(env):
    """The operators together: prompts of a best-effort client run as the profiler chooses beside a
    high-priority client's decode steps, whose prefix is a prompt's K and V; every output is what the calls
    give one after another."""
    B, ctx, torch = env
    heads, kv, dim, total = 8, 2, 128, 3000
    g = torch.Generator(device="cuda").manual_seed(2)
    qkv = torch.randn((total, heads + 2 * kv, dim), generator=g, device="cuda").to(torch.bfloat16)
    cu = torch.tensor([0, 1, 1500, total], dtype=torch.int32, device="cuda")
    out = torch.zeros((total, heads, dim), dtype=torch.bfloat16, device="cuda")
    prompt = B.attn_prompt_bf16(qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:], out, cu)
    step, results = _decode_step(B, torch, g, 5, heads, kv, dim, qkv[1500:, heads:], 30)
    torch.cuda.synchronize()
    ctx.launch_native(prompt)
    for kern in step:
        ctx.launch_native(kern, hi=True)
    torch.cuda.synchronize()
    want = [t.clone() for t in (out,) + results]
    assert all(torch.isfinite(t.float()).all() and t.float().abs().sum() > 0 for t in want)
    for t in (out,) + results:
        t.zero_()
    torch.cuda.synchronize()
    sched = ctx.scheduler()
    try:
        sched.submit_be(prompt, loop=True)
        sched.submit_be(step[1], (B.CFG_PTB, 16, 1), loop=False)   # (a product as best-effort work, too)
        for _ in range(40):
            sched.submit_hi(step)
            while sched.poll():
                pass
        import time
        t0 = time.perf_counter()
        while sched.stats()["be_kernels_done"] < 5 and time.perf_counter() - t0 < 20:
            time.sleep(0.001)
        assert sched.stats()["hi_requests_done"] == 40 and sched.stats()["be_kernels_done"] >= 5
    finally:
        sched.close()
    torch.cuda.synchronize()
    for name, a, b in zip(("prompt", "attention", "first product", "second product"), (out,) + results, want):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16)), name


def test_captured_decode_step_replays_beside_eager_work(env):
    """A captured decode step, replayed with the program's own work and waits between; new inputs in the
    same buffers give new outputs."""
    B, ctx, torch = env
    heads, kv, dim = 4, 1, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    shared = torch.randn((300, 2 * kv, dim), generator=g, device="cuda").to(torch.bfloat16)
    step, results = _decode_step(B, torch, g, 6, heads, kv, dim, shared, 40)
    prompt_in = torch.randn((200, heads, dim), generator=g, device="cuda").to(torch.bfloat16)
    prompt_out = torch.zeros_like(prompt_in)
    step = [B.attn_prompt_bf16(prompt_in, prompt_in, prompt_in, prompt_out, torch.tensor([0, 90, 200], dtype=torch.int32, device="cuda"))] + step
    results = (prompt_out,) + results
    torch.cuda.synchronize()
    for kern in step:
        ctx.launch_native(kern, hi=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=ctx._streams[0]):
        for kern in step:
            ctx.launch_native(kern, hi=True)
    for turn in range(4):
        shared.copy_(torch.randn(shared.shape, generator=g, device="cuda"))
        prompt_in.copy_(torch.randn(prompt_in.shape, generator=g, device="cuda"))
        torch.cuda.synchronize()
        for kern in step:
            ctx.launch_native(kern, hi=True)
        torch.cuda.synchronize()
        want = [t.clone() for t in results]
        for t in results:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(results, want):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16)), turn


def test_two_calls_at_once_on_two_streams(env):
    """Decode steps of two batches on the two streams, each with scratch of its own."""
    B, ctx, torch = env
    g = torch.Generator(device="cuda").manual_seed(4)
    shared = torch.randn((2000, 4, 128), generator=g, device="cuda").to(torch.bfloat16)
    steps = [_decode_step(B, torch, g, n, 8, 2, 128, shared, 300) for n in (3, 16)]
    torch.cuda.synchronize()
    want = []
    for kernels, results in steps:
        for kern in kernels:
            ctx.launch_native(kern, hi=True)
        torch.cuda.synchronize()
        want.append([t.clone() for t in results])
    for _ in range(10):
        for _, results in steps:
            for t in results:
                t.zero_()
        torch.cuda.synchronize()
        for pair in zip(*(kernels for kernels, _ in steps)):
            ctx.launch_native(pair[0], hi=True)
            ctx.launch_native(pair[1], hi=False)
        torch.cuda.synchronize()
        for (_, results), w in zip(steps, want):
            assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(results, w))


def test_measurements_of_calls_with_equal_grids_are_kept_apart(env):
    """The grid of a 4-bit product has n alone, a prompt's only heads, tokens and sequences: the profiler's records
    and choices are per sizes, and one call's are not another's."""
    B, ctx, torch = env
    z = lambda *s: torch.zeros(s, dtype=torch.int16, device="cuda")
    def product(m, k, group, zeros):
        W = torch.zeros((4, -(-k // 128), 64, 4), dtype=torch.int32, device="cuda")
        zp = torch.zeros((4, -(-k // group), 16), dtype=torch.uint8, device="cuda") if zeros else None
        return B.gemv_w4_bf16(z(m, k), W, z(4, -(-k // group), 16), z(m, 64), zeros=zp, group=group)
    def prompt(total, heads, kv, dim, seqs):
        cu = torch.tensor([total * i // seqs for i in range(seqs + 1)], dtype=torch.int32, device="cuda")
        return B.attn_prompt_bf16(z(total, heads, dim), z(total, kv, dim), z(total, kv, dim), z(total, heads, dim), cu)
    calls = [[product(*c) for c in ((1, 256, 64, False), (2, 256, 64, False), (1, 1024, 64, False), (1, 256, 32, False), (1, 256, 64, True))],
             [prompt(*c) for c in ((300, 4, 4, 64, 2), (300, 4, 4, 128, 2), (300, 4, 2, 64, 2), (200, 4, 4, 64, 3), (300, 2, 2, 64, 6))]]
    ctx.profile_reset()
    torch.cuda.synchronize()
    for same in calls:
        for i, kern in enumerate(same):
            assert kern.desc.grid.x == same[0].desc.grid.x
            for later in same[i:]:
                assert ctx.profile_table(later) == ([], -1)
                assert ctx.lookup_config(later) is None
            ctx.profile(kern, [(B.CFG_PTB, 4, 1), (B.CFG_SLICED, 1 + i, 1)], runs=1)
            assert all(len(ctx.profile_table(k)[0]) == 2 for k in same[:i + 1])
        assert [ctx.profile_table(k)[0][1]["param"] for k in same] == [1 + i for i in range(len(same))]
    assert len(ctx.profile_table(prompt(280, 4, 4, 64, 2))[0]) == 2   # (20 tokens fewer: the same blocks, nearly the same time)
    ctx.profile_reset()


def test_footprints_leave_room_for_a_paused_product(env):
    """The 4-bit products fit beside a paused 256 x 256 GEMM tile (their eight waves are compiled for 72 registers
    except with four rows of tiles), and what the prompt's workers occupy is known to the admission rules."""
    B, ctx, _ = env
    lds, waves, regs = ctx.kernel_footprint(B.K_GEMM_BF16, 0)
    whole = B.device_info()["lds_bytes_per_cu"]
    l4, w4, r4 = ctx.kernel_footprint(B.K_GEMV_W4_BF16, 1)
    assert lds + l4 <= whole and w4 == 8 and r4 <= 96 and regs + 2 * 72 <= 512
    lp, wp, rp = ctx.kernel_footprint(B.K_ATTN_PROMPT_BF16, 0)
    assert 2 * lp <= whole and wp == 4 and rp <= 256
