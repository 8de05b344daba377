"""CPU-side checks of rotary positions and the paged cache: logical grids, refusals, layouts.  No kernel runs."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import paged as OP

P = 4096                                                   # any 16-byte aligned address: nothing is read


@pytest.fixture(scope="module")
def B():
    import paper_2410_07381_amd.binding as B
    return B


def _rope(B, **other):
    return B.RopeArgs(**dict(dict(x=P, out=P, freqs=P, positions=P, total=1000, heads=8, dim=128, rot=64), **other))


def _append(B, **other):
    a = dict(k=P, v=P, cu_seqlens=P, lens=P, table=P, freqs=P, positions=P, k_pages=P, v_pages=P, k_exps=P, v_exps=P, total=1000, n_seqs=3,
             kv_heads=2, dim=128, page=16, n_pages=100, seq_pages=40, rot=64)
    return B.KvAppendArgs(**dict(a, **other))


def _paged(B, **other):
    a = dict(q=P, out=P, k_pages=P, v_pages=P, k_exps=P, v_exps=P, table=P, lens=P, scratch=P, batch=3, heads=8, kv_heads=2, dim=128, page=16,
             n_pages=100, seq_pages=40)
    return B.AttnPagedArgs(**dict(a, **other))


def test_struct_sizes(B):
    assert C.sizeof(B.RopeArgs) == 64 and C.sizeof(B.KvAppendArgs) == 144 and C.sizeof(B.AttnPagedArgs) == 120


def _refused(B, kernel, args):
    with pytest.raises(B.TallyError) as e:
        B.logical_grid(kernel, args)
    assert e.value.status == B.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(out=None), dict(freqs=None), dict(positions=None), dict(x=P + 8), dict(out=P + 4), dict(freqs=P + 2), dict(positions=P + 1),
    dict(total=0), dict(total=(1 << 30) + 1), dict(total=1 << 30, heads=64), dict(heads=0), dict(heads=1 << 14), dict(dim=0), dict(dim=72), dict(dim=528),
    dict(rot=0), dict(rot=8), dict(rot=144), dict(ld_x=1016), dict(ld_x=1028), dict(ld_out=(1 << 20) + 8), dict(flags=4), dict(magnitude=-1.0),
    dict(magnitude=65.0), dict(magnitude=float("nan")), dict(magnitude=float("inf"))])
def test_rope_refusals(B, bad):
    _refused(B, B.K_ROPE_BF16, _rope(B, **bad))


@pytest.mark.parametrize("total,heads,dim,rot", [(1, 1, 16, 16), (5, 40, 128, 128), (1000, 1, 64, 64), (100000, 1, 64, 64), (100000, 1, 512, 512), (32768, 40, 128, 128)])
def test_rope_blocks_hold_a_table_and_cover_every_token(B, total, heads, dim, rot):
    blocks = B.logical_grid(B.K_ROPE_BF16, _rope(B, total=total, heads=heads, dim=dim, rot=rot))[0][0]
    tokens = [g for g in (1, 2, 4, 8, 16, 32) if -(-total // g) == blocks]
    assert tokens and min(tokens) * rot // 2 <= 2048


@pytest.mark.parametrize("bad", [
    dict(k=None), dict(v=None), dict(cu_seqlens=None), dict(lens=None), dict(table=None), dict(freqs=None), dict(k_pages=None), dict(v_pages=None),
    dict(k_exps=None), dict(v_exps=None), dict(k=P + 8), dict(v=P + 2), dict(k_pages=P + 8), dict(v_pages=P + 1), dict(cu_seqlens=P + 2), dict(lens=P + 2),
    dict(table=P + 3), dict(freqs=P + 2), dict(positions=P + 2), dict(total=0), dict(total=(1 << 30) + 1), dict(n_seqs=0), dict(n_seqs=(1 << 24) + 1), dict(n_seqs=1 << 24, kv_heads=16), dict(kv_heads=0),
    dict(kv_heads=1 << 17), dict(dim=96), dict(dim=256), dict(page=0), dict(page=8), dict(page=48), dict(page=256), dict(n_pages=0), dict(n_pages=(1 << 30) + 1),
    dict(seq_pages=0), dict(seq_pages=(1 << 24) + 1), dict(ld_table=39), dict(ld_k=248), dict(ld_k=260), dict(ld_v=(1 << 20) + 8), dict(rot=8), dict(rot=144),
    dict(flags=2), dict(flags=4), dict(magnitude=-0.5), dict(magnitude=float("nan")), dict(total=1 << 30, kv_heads=16), dict(total=1 << 30, kv_heads=64, page=128)])
def test_append_refusals(B, bad):
    _refused(B, B.K_KV_APPEND_FP8, _append(B, **bad))


def test_append_without_turning_does_not_look_at_its_pointers(B):
    assert B.logical_grid(B.K_KV_APPEND_FP8, _append(B, rot=0, freqs=None, positions=P + 2))[0] == (34 * 2, 1, 1)
    assert B.logical_grid(B.K_KV_APPEND_FP8, _append(B, positions=None))[0] == (34 * 2, 1, 1)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_append_grid_has_room_for_every_sequence(B, page, dim):
    """Sequence s has the slots from cu[s] / page + 2 s up to the next one's: enough wherever its tokens begin in a page.  The grid
    has all slots, some of them side by side in a block, and all heads, up to four of them one after the other."""
    rng = np.random.default_rng(page)
    for kv in (1, 2, 3, 8, 24):
        for n, most in ((1, 4 * page), (7, 4 * page), (300, 4 * page), (300, 2), (300, 4), (40, 12), (1, 200000)):
            new = rng.integers(0, most, n) * (rng.random(n) < 0.7)
            cu = np.concatenate([[0], np.cumsum(new)])
            total = max(int(cu[-1]), 1)
            grid, block = B.logical_grid(B.K_KV_APPEND_FP8, _append(B, total=total, n_seqs=n, kv_heads=kv, page=page, dim=dim))
            # a page and head has pieces: a wave each; or, with hardly more than a token a sequence, one wave for all of them, or
            # (of more than four) four waves
            pieces = page * dim // 1024
            kind = 1 if total <= n + n // 8 else 4 if pieces > 4 and total < n * page // 8 else 0
            waves = 4 if kind else max(4, pieces)
            together = 4 // kind if kind else waves // pieces
            assert block == (64 * waves, 1, 1) and grid[1:] == (1, 1)
            by_slots = -(-(total // page + 2 * n) // together)
            assert grid[0] % by_slots == 0 and grid[0] // by_slots in {-(-kv // h) for h in ((1,) if kind else (1, 2, 4)) if h <= kv}
            start = cu // page + 2 * np.arange(n + 1)
            for at in range(page):                         # the first new token's place in its page
                pages = np.where(new > 0, (at + new - 1) // page + 1, 0)
                assert (pages <= np.diff(start)).all()


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(out=None), dict(k_pages=None), dict(v_pages=None), dict(k_exps=None), dict(v_exps=None), dict(table=None), dict(lens=None), dict(scratch=None),
    dict(q=P + 8), dict(out=P + 2), dict(k_pages=P + 8), dict(v_pages=P + 4), dict(table=P + 2), dict(lens=P + 1), dict(scratch=P + 8), dict(batch=0),
    dict(batch=1 << 18), dict(heads=9), dict(heads=0), dict(kv_heads=0), dict(kv_heads=16), dict(dim=80), dict(page=8), dict(page=96), dict(n_pages=0),
    dict(n_pages=(1 << 30) + 1), dict(seq_pages=0), dict(seq_pages=(1 << 24) + 1), dict(batch=1 << 10, seq_pages=(1 << 22) + 1), dict(ld_table=39), dict(ld_q=1016),
    dict(ld_q=1028), dict(ld_out=1000), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))])
def test_attention_refusals(B, bad):
    _refused(B, B.K_ATTN_PAGED_FP8, _paged(B, **bad))


def test_attention_scratch(B):
    """None where no sequence can have two parts, else a record for every part that there may be, acc from a multiple of 16 bytes on."""
    assert B.attn_paged_scratch_bytes(3, 8, 2, 128, 16, 1) == 0
    assert B.logical_grid(B.K_ATTN_PAGED_FP8, _paged(B, seq_pages=1, scratch=None))[0] == (8, 3, 1)
    for refused in ((0, 8, 2, 128, 16, 4), (3, 8, 3, 128, 16, 4), (3, 8, 2, 96, 16, 4), (3, 8, 2, 128, 24, 4), (3, 8, 2, 128, 16, 0), (1 << 20, 2, 2, 64, 16, 4)):
        assert B.attn_paged_scratch_bytes(*refused) == 0
    for batch, heads, kv, dim, page, pages in ((1, 1, 1, 64, 16, 200), (3, 7, 1, 64, 32, 1000), (64, 32, 8, 128, 128, 1024)):
        size = B.attn_paged_scratch_bytes(batch, heads, kv, dim, page, pages)
        slots = next(s for s in range(1, 2000) if -(-s * heads * 2 // 4) * 16 + s * heads * dim * 4 >= size)
        assert -(-slots * heads * 2 // 4) * 16 + slots * heads * dim * 4 == size


@pytest.mark.parametrize("page,dim", [(16, 64), (64, 128)])
def test_the_cache_holds_what_its_layout_says(B, page, dim):
    import torch
    rng = np.random.default_rng(page)
    c = OP.empty_cache(3, 2, page, dim)
    for n in ("k", "v"):
        c[n] = rng.integers(0, 256, c[n].shape).astype(np.uint8)
        c[n][(c[n] & 127) == 127] = 0
        c[n + "_exps"] = rng.integers(1, 255, c[n + "_exps"].shape).astype(np.uint8)
    cache = B.PagedCache(*(torch.from_numpy(c[n]) for n in ("k", "v", "k_exps", "v_exps")))
    for name, got in zip(("k", "v"), cache.values()):
        for p in range(3):
            want, there = OP.tokens_of(c, name, [p], page)
            assert there.all() and (got[p].transpose(0, 1).numpy() == want.astype(np.float32)).all()
    empty = B.PagedCache.empty(5, 2, page, dim, device="cpu")
    assert [tuple(t.shape) for t in empty] == [(5, 2, page, dim), (5, 2, page // 16, dim, 16), (5, 2), (5, 2)]


def test_frequencies(B):
    f, m = B.rope_freqs(8)
    assert m == 1.0 and f.dtype.is_floating_point and np.allclose(f.numpy(), [1, 0.1, 0.01, 0.001], rtol=1e-6)
    assert np.allclose(B.rope_freqs(8, factor=4.0)[0].numpy(), f.numpy() / 4)
    base = B.rope_freqs(8, factor=4.0, scaling="base")[0].numpy()
    assert base[0] == 1 and base[-1] == pytest.approx(0.001 / 4, rel=1e-6)
    parts, m = B.rope_freqs(8, factor=4.0, scaling="parts", context=1000, turns=(1.0, 20.0))
    turns = 1000 * f.numpy().astype(float) / (2 * math.pi)   # 159, 15.9, 1.59, 0.159
    keep = np.clip((turns - 1) / 19, 0, 1)
    assert keep[0] == 1 and keep[-1] == 0 and np.allclose(parts.numpy(), f.numpy() * (keep + (1 - keep) / 4)) and m == pytest.approx(0.1 * math.log(4) + 1)
    for bad in (dict(rot=7), dict(rot=0), dict(rot=8, factor=0.5), dict(rot=8, scaling="other"), dict(rot=8, scaling="parts"), dict(rot=2, scaling="base", factor=2.0)):
        with pytest.raises(AssertionError):
            B.rope_freqs(**bad)


def test_the_binding_checks_shapes_types_and_strides(B):
    import torch
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32)
    x, f, at = z(5, 4, 64), torch.ones(16), ints(0, 1, 2, 3, 4)
    B.rope_bf16(x, x, f, at)
    B.rope_bf16(z(5, 9, 64)[:, 2:6], x, f, at, interleaved=True, inverse=True, magnitude=1.5)
    for args in ((x, x[:4], f, at), (x.float(), x, f, at), (x.half(), x, f, at), (x, x, f.double(), at), (x, x, f, at.long()), (x, x, f, at[:4]),
                 (x[:, ::2], x[:, ::2], f, at), (x, x, f[::2], at), (x[:1].expand(5, 4, 64), x, f, at)):
        with pytest.raises(AssertionError):
            B.rope_bf16(*args)
    for bad in (0.0, -1.0):
        with pytest.raises(AssertionError):
            B.rope_bf16(x, x, f, at, magnitude=bad)
    with pytest.raises(B.TallyError):
        B.rope_bf16(x, x, torch.ones(36), at)
    cache = B.PagedCache.empty(6, 4, 16, 64, device="cpu")
    cu, lens, table = ints(0, 2, 5), ints(9, 20), torch.zeros((2, 3), dtype=torch.int32)
    good = (x, x, cu, lens, table, cache)
    B.kv_append_fp8(*good)
    B.kv_append_fp8(*good, freqs=f, positions=at)
    B.kv_append_fp8(*good[:5], B.PagedCache(*(t.view(torch.float8_e4m3fn) for t in cache[:2]), *cache[2:]))
    swap = lambda i, v: tuple(v if j == i else g for j, g in enumerate(good))
    other = lambda **k: cache._replace(**k)
    for args in (swap(0, x[:4]), swap(0, x.float()), swap(1, x.half()), swap(2, cu.long()), swap(2, cu[:1]), swap(3, lens[:1]), swap(3, lens.float()),
                 swap(4, table[:1]), swap(4, table.long()), swap(4, table[:, :0]), swap(4, torch.zeros((2, 6), dtype=torch.int32)[:, ::2]),
                 swap(5, other(k=cache.k.to(torch.int8))), swap(5, other(k=cache.k[:, :2])), swap(5, other(v=cache.v.transpose(3, 4))),
                 swap(5, other(k_exps=cache.k_exps[:5])), swap(5, other(v_exps=cache.v_exps.to(torch.int32))), swap(5, B.PagedCache.empty(6, 2, 16, 64, device="cpu"))):
        with pytest.raises(AssertionError):
            B.kv_append_fp8(*args)
    for bad in (dict(freqs=f.double()), dict(positions=at), dict(freqs=f, positions=at[:3]), dict(freqs=f, magnitude=0.0)):
        with pytest.raises(AssertionError):
            B.kv_append_fp8(*good, **bad)
    q, out = z(2, 8, 64), z(2, 8, 64)
    assert B.attn_paged_scratch_bytes(2, 8, 4, 64, 16, 3) == 0
    B.attn_paged_fp8(q, cache, table, lens, out)
    wide = torch.zeros((2, 100), dtype=torch.int32)
    room = torch.zeros(B.attn_paged_scratch_bytes(2, 8, 4, 64, 16, 100), dtype=torch.uint8)
    assert room.numel() > 0
    B.attn_paged_fp8(q, cache, wide, lens, out, room, scale=0.5)
    for args in ((q, cache, wide, lens, out), (q, cache, wide, lens, out, room[:-1]), (q, cache, table[:1], lens, out), (q, cache, table, lens.long(), out),
                 (q, cache, table, lens[:1], out), (q[:, :, :32], cache, table, lens, out[:, :, :32]), (q, cache, table, lens, out[:1]), (q.half(), cache, table, lens, out)):
        with pytest.raises(AssertionError):
            B.attn_paged_fp8(*args)
    with pytest.raises(AssertionError):
        B.attn_paged_fp8(q, cache, table, lens, out, scale=0.0)
    with pytest.raises(B.TallyError):
        B.attn_paged_fp8(q[:, :7], cache, table, lens, out[:, :7])


def test_registers_leave_room_beside_a_paused_tile(B, tmp_path):
    """Attention over pages: 128 registers and 31 KB of LDS at most, so that a workgroup fits beside a paused 256 x 256 GEMM tile."""
    import re
    from test_host_logic import _device_code
    notes = _device_code(B, tmp_path)("llvm-readelf", "--notes")
    found = {}
    for kernel in notes.split("- .agpr_count:")[1:]:
        name, regs = re.search(r"\.name:\s+(_Z\S+)", kernel), re.search(r"\.vgpr_count:\s+(\d+)", kernel)
        lds, spilled = re.search(r"\.group_segment_fixed_size:\s+(\d+)", kernel), re.search(r"\.private_segment_fixed_size:\s+(\d+)", kernel)
        found[name.group(1)] = (int(regs.group(1)) + int(kernel.split()[0]), int(lds.group(1)), int(spilled.group(1)))
    mine = {n: r for n, r in found.items() if "attn_paged" in n}
    assert len(mine) == 12 and all(r[0] <= 128 and r[1] <= 31 * 1024 for r in mine.values()), mine
    # nothing in memory beside the registers, but what the workers of sixteen waves miss of 128
    rest = {n: r for n, r in found.items() if "attn_paged" in n or "RopeBody" in n or "AppendBodyT" in n}
    assert len(rest) == 12 + 3 + 27 and all(r[2] <= (16 if "ptb" in n and "ELi16E" in n else 0) for n, r in rest.items()), rest
