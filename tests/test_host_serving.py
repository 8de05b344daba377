"""CPU-side checks of the serving operators: logical grids, refusals, layouts.  No kernel runs."""
import ctypes as C

import numpy as np
import pytest

from oracle import serving as OS

P = 4096                                                   # any 16-byte aligned address: nothing is read


@pytest.fixture(scope="module")
def B():
    import paper_2410_07381_amd.binding as B
    return B


def _prompt(B, **other):
    a = dict(q=P, k=P, v=P, out=P, cu_seqlens=P, total=1000, n_seqs=3, heads=8, kv_heads=2, dim=128, scale=0.0)
    return B.AttnPromptArgs(**dict(a, **other))


def _prefix(B, **other):
    a = dict(q=P, K=P, V=P, Ko=P, Vo=P, own_len=P, out=P, scratch=P, batch=3, prefix=100, own_cap=50, heads=8,
             kv_heads=2, dim=128, scale=0.0)
    return B.AttnPrefixArgs(**dict(a, **other))


def _w4(B, **other):
    a = dict(x=P, W=P, scales=P, zeros=P, y=P, m=4, n=100, k=256, group=64)
    return B.GemvW4Args(**dict(a, **other))


def test_struct_sizes(B):
    assert C.sizeof(B.AttnPromptArgs) == 80 and C.sizeof(B.AttnPrefixArgs) == 120 and C.sizeof(B.GemvW4Args) == 64


@pytest.mark.parametrize("total,seqs,heads", [(1, 1, 1), (127, 1, 2), (128, 1, 2), (1000, 3, 8), (1 << 26, 1 << 20, 8)])
def test_prompt_grid_has_room_for_every_sequence(B, total, seqs, heads):
    grid, block = B.logical_grid(B.K_ATTN_PROMPT_BF16, _prompt(B, total=total, n_seqs=seqs, heads=heads, kv_heads=1))
    assert block == (256, 1, 1) and grid[0] % heads == 0 and grid[1:] == (1, 1)
    # sequence s has the slots from cu[s] / 128 + s up to the next one's: enough wherever it begins
    rng = np.random.default_rng(total)
    cu = np.sort(rng.integers(0, total + 1, min(seqs, 1000) + 1))
    slots = cu // 128 + np.arange(len(cu))
    assert (np.diff(slots) >= -(-np.diff(cu) // 128)).all() and (np.diff(slots) <= np.diff(cu) // 128 + 2).all()
    assert cu[-1] // 128 + seqs <= grid[0] // heads


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(cu_seqlens=None), dict(q=P + 8), dict(k=P + 2),
    dict(v=P + 4), dict(out=P + 8), dict(cu_seqlens=P + 2), dict(total=0), dict(total=(1 << 30) + 1), dict(n_seqs=0),
    dict(n_seqs=1 << 21), dict(total=1 << 28),
    dict(heads=0), dict(kv_heads=0), dict(heads=7), dict(kv_heads=16), dict(dim=96), dict(dim=0), dict(dim=256),
    dict(ld_q=1016), dict(ld_q=1028), dict(ld_k=255), dict(ld_v=128), dict(ld_out=(1 << 20) + 8), dict(scale=-1.0),
    dict(scale=float("nan")), dict(scale=float("inf"))])
def test_prompt_refusals(B, bad):
    with pytest.raises(B.TallyError) as e:
        B.logical_grid(B.K_ATTN_PROMPT_BF16, _prompt(B, **bad))
    assert e.value.status == B.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(out=None), dict(scratch=None), dict(K=None), dict(V=None), dict(Ko=None), dict(Vo=None),
    dict(own_len=None), dict(q=P + 8), dict(K=P + 8), dict(Vo=P + 8), dict(own_len=P + 1), dict(scratch=P + 8),
    dict(batch=0), dict(batch=1 << 20), dict(prefix=(1 << 28) + 1), dict(own_cap=(1 << 28) + 1), dict(heads=9),
    dict(kv_heads=0), dict(dim=80), dict(ld_q=1000), dict(ld_prefix=264 - 16), dict(ld_own=260), dict(ld_out=1016),
    dict(stride_own=4), dict(stride_own=50 * 256 - 8), dict(scale=-0.5), dict(scale=float("nan"))])
def test_prefix_refusals(B, bad):
    with pytest.raises(B.TallyError) as e:
        B.logical_grid(B.K_ATTN_PREFIX_BF16, _prefix(B, **bad))
    assert e.value.status == B.ERR_INVALID_ARG


def test_prefix_without_a_part_does_not_look_at_its_pointers(B):
    for a in (_prefix(B, prefix=0, K=None, V=None), _prefix(B, own_cap=0, Ko=None, Vo=None, own_len=None),
              _prefix(B, prefix=0, own_cap=0, K=None, V=None, Ko=None, Vo=None, own_len=None, scratch=None)):
        assert B.logical_grid(B.K_ATTN_PREFIX_BF16, a)[0] == (8, 3, 1)
    assert B.attn_prefix_scratch_bytes(3, 8, 2, 128, 0, 0) == 0
    assert B.attn_prefix_scratch_bytes(3, 8, 2, 128, 1, 0) == 3 * 8 * 130 * 4
    for refused in ((0, 8, 2, 128, 1, 1), (3, 8, 3, 128, 1, 1), (3, 8, 2, 72, 1, 1), (1 << 20, 8, 2, 128, 1, 1)):
        assert B.attn_prefix_scratch_bytes(*refused) == 0


@pytest.mark.parametrize("batch,heads,kv,dim,prefix,cap", [(32, 32, 8, 128, 4096, 512), (64, 32, 8, 128, 65500, 1024), (24, 32, 8, 64, 2000, 500)])
def test_prefix_is_cut_up_like_its_neighbours(B, batch, heads, kv, dim, prefix, cap):
    """One token more or less in the prefix or in the caches does not move a call across a line of the plan."""
    def parts(p, c):
        n = B.attn_prefix_scratch_bytes(batch, heads, kv, dim, p, c)
        return n // (batch * heads * (dim * 4 + 8))
    assert {parts(p, c) for p in (prefix - 1, prefix, prefix + 1) for c in (cap - 1, cap)} == {parts(prefix, cap)}


@pytest.mark.parametrize("batch,heads,kv,dim,prefix,cap,records", [(1, 7, 1, 128, 4000, 64, 231), (1, 1, 1, 64, 300, 0, 3),
                                                                   (3, 5, 5, 64, 2000, 0, 240), (1, 7, 1, 128, 3968, 128, 224)])
def test_prefix_scratch_keeps_the_weighted_sums_aligned(B, batch, heads, kv, dim, prefix, cap, records):
    """A record of (max, sum) for each row's parts, then from a multiple of 16 bytes on, with odd numbers of them too,
    the parts' weighted sums, which are read and written 16 bytes at a time."""
    assert B.attn_prefix_scratch_bytes(batch, heads, kv, dim, prefix, cap) == -(-records * 8 // 16) * 16 + records * dim * 4


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(W=None), dict(scales=None), dict(y=None), dict(x=P + 8), dict(W=P + 4), dict(m=0), dict(m=17),
    dict(n=0), dict(k=0), dict(k=252), dict(group=0), dict(group=16), dict(group=96), dict(group=192), dict(ld_x=248),
    dict(ld_x=260), dict(ld_y=99)])
def test_w4_refusals(B, bad):
    with pytest.raises(B.TallyError) as e:
        B.logical_grid(B.K_GEMV_W4_BF16, _w4(B, **bad))
    assert e.value.status == B.ERR_INVALID_ARG


@pytest.mark.parametrize("m,n,rows", [(1, 1, 1), (1, 16384, 1), (2, 16385, 2), (4, 4096, 1), (4, 11008, 2), (8, 11008, 3), (8, 16384, 2),
                                      (16, 4096, 1), (16, 11008, 3), (16, 16384, 2), (16, 32000, 4), (16, 50256, 4), (5, 50257, 2)])
def test_w4_rows_of_tiles_by_vectors_and_rows(B, m, n, rows):
    """The rule's measured best: workgroups of as many rows as keep x from being read again and again, with the
    same number of workgroups on every compute unit."""
    assert B.logical_grid(B.K_GEMV_W4_BF16, _w4(B, m=m, n=n))[0] == (-(-n // (16 * rows)), 1, 1)


def test_w4_grid_and_optional_zeros(B):
    assert B.logical_grid(B.K_GEMV_W4_BF16, _w4(B, zeros=None))[0] == (7, 1, 1)
    assert B.logical_grid(B.K_GEMV_W4_BF16, _w4(B, n=112, k=8, group=256))[0] == (7, 1, 1)


@pytest.mark.parametrize("n,k", [(1, 8), (16, 128), (37, 264), (50, 1000)])
def test_pack_w4_lays_out_what_the_header_says(B, n, k):
    import torch
    rng = np.random.default_rng(n)
    codes = rng.integers(0, 16, (n, k))
    W = B.pack_w4(torch.from_numpy(codes))
    assert W.dtype == torch.int32 and W.shape == (-(-n // 16), -(-k // 128), 64, 4)
    assert (OS.w4_codes(W.numpy(), n, k) == codes).all()
    full = OS.w4_codes(W.numpy(), W.shape[0] * 16, W.shape[1] * 128)
    assert full[n:].sum() == 0 and full[:, k:].sum() == 0
    t = torch.arange(n * 3, dtype=torch.float32).view(n, 3)
    g = B.pack_w4_groups(t)
    assert g.shape == (W.shape[0], 3, 16)
    assert all(g[r // 16, j, r % 16] == t[r, j] for r in range(n) for j in range(3))


def test_the_binding_checks_shapes_and_strides(B):
    import torch
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    cu = torch.tensor([0, 5], dtype=torch.int32)
    q, kv = z(5, 4, 64), z(5, 4, 64)
    B.attn_prompt_bf16(q, kv[:, :2], kv[:, 2:], z(5, 4, 64), cu)
    for args in ((q, kv[:, :2], kv[:, 1:], q, cu), (q[:, :, ::2], q, q, q, cu), (q, kv[:, ::2], kv[:, ::2], q, cu),
                 (q, z(1, 2, 64).expand(5, 2, 64), kv[:, :2], q, cu), (q.float(), kv, kv, q, cu),
                 (q, kv, kv, q, cu.long()), (q, kv, kv, q, cu[:1])):
        with pytest.raises(AssertionError):
            B.attn_prompt_bf16(*args)
    with pytest.raises(AssertionError):
        B.attn_prompt_bf16(q, kv, kv, z(5, 4, 64), cu, scale=0.0)
    own, lens = z(3, 7, 2, 64), torch.zeros(3, dtype=torch.int32)
    room = torch.zeros(B.attn_prefix_scratch_bytes(3, 4, 2, 64, 5, 7), dtype=torch.uint8)
    q3 = z(3, 4, 64)
    B.attn_prefix_bf16(q3, kv[:, :2], kv[:, 2:], own, own, lens, z(3, 4, 64), room)
    for args in ((q3, kv[:, :2], z(5, 2, 64), own, own, lens, q3, room), (q3, kv[:, :2], kv[:, 2:], own, own[:, :6], lens, q3, room),
                 (q3, kv[:, :2], kv[:, 2:], own, own, lens[:2], q3, room), (q3, kv[:, :2], kv[:, 2:], own, own, lens, q3, room[:-4]),
                 (q3, kv[:, :2], kv[:, 2:], own[:1].expand(3, 7, 2, 64), own[:1].expand(3, 7, 2, 64), lens, q3, room)):
        with pytest.raises(AssertionError):
            B.attn_prefix_bf16(*args)
    x, y = z(2, 256), z(2, 20)
    W, s = B.pack_w4(torch.zeros(20, 256, dtype=torch.uint8)), z(2, 2, 16)
    B.gemv_w4_bf16(x, W, s, y)
    for args in ((x, W[:1], s, y), (x, W, s[:, :1], y), (x, W, s, y[:1]), (z(2, 512)[:, ::2], W, s, y),
                 (x[:1].expand(2, 256), W, s, y)):
        with pytest.raises(AssertionError):
            B.gemv_w4_bf16(*args)


@pytest.fixture(scope="module")
def estimate(tmp_path_factory):
    """The turnaround estimate of prompts as workers: for every (latency us, workers, chunk, looks every, heads, total, n_seqs)."""
    import os
    import subprocess
    src = tmp_path_factory.mktemp("turnaround") / "turnaround.cpp"
    src.write_text(r"""
#include <cstdio>
#include "turnaround.h"
using namespace tally;
int main() {
  tally_attn_prompt_args a{};
  double us;
  uint32_t workers, chunk, every;
  while (scanf("%lf %u %u %u %u %u %u", &us, &workers, &chunk, &every, &a.heads, &a.total, &a.n_seqs) == 7)
    printf("%.9g\n", 1e3 * workers_turnaround_ms(us * 1e-3, workers, chunk, (uint64_t)a.heads * prompt_slots(a), prompt_pause_share(a, every)));
  return 0;
}
""")
    exe = src.with_suffix("")
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_07381_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", csrc, str(src), "-o", str(exe)], check=True, timeout=60)
    return lambda *c: float(subprocess.run([str(exe)], input=" ".join(map(str, c)), capture_output=True, text=True, check=True).stdout)


def _tiles(lens):
    """Tiles of the blocks of one head."""
    return [-(-min(r + 128, n) // 64) for n in lens for r in range(0, n, 128)]


@pytest.mark.parametrize("every", [1, 4, 16])
@pytest.mark.parametrize("total", [1, 64, 128, 129, 1000, 4097, 32768])
def test_prompt_turnaround_of_one_sequence_is_that_of_the_tiles_between_two_looks(estimate, total, every):
    """A worker hands over `every` + 1 tiles after the request, or at its block's end; a tile's time is the kernel's over
    the tiles that each worker has."""
    heads, workers = 8, 256
    tiles = _tiles([total])
    tile_us = 1000.0 * workers / (heads * sum(tiles))
    slots = total // 128 + 1
    want = min(every + 1, sum(tiles) / slots) * tile_us
    assert estimate(1000.0, workers, 1, every, heads, total, 1) == pytest.approx(want, rel=1e-6)
    chunk = 16 if want == sum(tiles) / slots * tile_us else 1   # (that stop between blocks alone: all of a fetch)
    assert estimate(1000.0, workers, 16, every, heads, total, 1) == pytest.approx(chunk * want, rel=1e-6)


@pytest.mark.parametrize("lens", [[int(4096 ** (i / 23) + 0.5) for i in range(24)], [256] * 64, [3000, 1], [8192] * 4])
def test_prompt_turnaround_of_several_sequences_is_not_that_of_one_of_all_tokens(estimate, lens):
    """Which blocks pause at all depends on lengths that the host does not know: the estimate is Eq. 1's, no shorter than
    the time of an average slot, whatever the number of blocks a fetch brings."""
    heads, workers, every = 32, 512, 4
    tiles = _tiles(lens)
    tile_us = 1000.0 * workers / (heads * sum(tiles))
    slots = sum(lens) // 128 + len(lens)
    for chunk in (1, 4):
        got = estimate(1000.0, workers, chunk, every, heads, sum(lens), len(lens))
        assert got == pytest.approx(chunk * sum(tiles) / slots * tile_us, rel=1e-6)


def test_registers_leave_the_room_that_the_kernels_count_on(B, tmp_path):
    """From the library's own notes, kernel by kernel: 4-bit products of one to three rows of tiles have 72 registers at most in
    every form (two of their eight waves fit beside a paused 256 x 256 tile's), those of four 96; attention behind a prefix in
    parts of 16 and 64 rows 128; prompts 256."""
    import re
    from test_host_logic import _device_code
    notes = _device_code(B, tmp_path)("llvm-readelf", "--notes")
    found = {}
    for kernel in notes.split("- .agpr_count:")[1:]:
        name, regs = re.search(r"\.name:\s+(_Z\S+)", kernel), re.search(r"\.vgpr_count:\s+(\d+)", kernel)
        found[name.group(1)] = int(regs.group(1)) + int(kernel.split()[0])
    w4 = {(m.group(1), int(m.group(2)), int(m.group(3))): r for n, r in found.items()
          if (m := re.search(r"(native|sliced|ptb)_kernelINS_7GemvW4TILi(\d)ELi(\d)E", n))}
    assert len(w4) == 36
    assert all(r <= (96 if rows == 4 else 72) for (_, _, rows), r in w4.items()), w4
    staged = {n: r for n, r in found.items() if "GemvW4StagedT" in n}
    assert len(staged) == 9 and max(staged.values()) <= 72
    behind = {(int(m.group(1)), int(m.group(2))): r for n, r in found.items()
              if (m := re.search(r"attn_prefix_partialILi(\d+)ELi(\d)E", n))}
    assert len(behind) == 6 and all(r <= (256 if kind == 2 else 128) for (_, kind), r in behind.items()), behind
    prompts = {n: r for n, r in found.items() if "PromptBodyT" in n}
    assert len(prompts) == 6 and max(prompts.values()) <= 256


def test_the_binding_refuses_types_that_would_be_taken_for_others(B):
    """fp16 for bf16, floats or 64 bits for lengths, codes of more than four bits, zero points above 128, groups of none."""
    import torch
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)
    half = lambda t: t.to(torch.float16)
    cu, q, lens = torch.tensor([0, 5], dtype=torch.int32), z(5, 2, 64), torch.zeros(3, dtype=torch.int32)
    q3, own = z(3, 2, 64), z(3, 7, 2, 64)
    room = torch.zeros(B.attn_prefix_scratch_bytes(3, 2, 2, 64, 5, 7), dtype=torch.uint8)
    x, y, W, s = z(2, 256), z(2, 20), B.pack_w4(torch.zeros(20, 256, dtype=torch.uint8)), z(2, 2, 16)
    calls = [(B.attn_prompt_bf16, (q, q, q, z(5, 2, 64), cu), range(4), 4), (B.attn_prefix_bf16, (q3, q, q, own, own, lens, z(3, 2, 64), room), (0, 1, 2, 3, 4, 6), 5),
             (B.gemv_w4_bf16, (x, W, s, y), (0, 2, 3), None)]
    for call, args, values, lengths in calls:
        call(*args)
        call(*(a.view(torch.int16) if i in values else a for i, a in enumerate(args)))
        bad = [(i, half(args[i])) for i in values] + ([(lengths, args[lengths].float()), (lengths, args[lengths].long())] if lengths else [])
        for i, other in bad:
            with pytest.raises(AssertionError):
                call(*args[:i], other, *args[i + 1:])
    with pytest.raises(AssertionError):
        B.gemv_w4_bf16(x, W, s, y, group=0)
    for codes in (torch.tensor([[16] * 8]), torch.tensor([[-1] * 8]), torch.ones(1, 8)):
        with pytest.raises(AssertionError):
            B.pack_w4(codes)
    for kind in (torch.uint8, torch.int8, torch.int16, torch.uint16, torch.int32, torch.uint32, torch.int64):
        assert (B.pack_w4(torch.full((1, 8), 15).to(kind))[0, 0, 0] == torch.tensor([-1, 0, 0, 0])).all()
    assert B.pack_w4_groups(torch.full((3, 2), 128, dtype=torch.uint8)).max() == 128
    with pytest.raises(AssertionError):
        B.pack_w4_groups(torch.full((3, 2), 129, dtype=torch.uint8))
