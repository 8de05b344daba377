"""CPU-side checks of rotary positions and the paged cache beside those of test_host_paged.py.  No kernel runs."""
import pytest


@pytest.fixture(scope="module")
def B():
    import paper_2410_07381_amd.binding as B
    return B


def test_tensors_on_different_devices_are_refused(B):
    """rope_freqs gives them on the host unless it is told otherwise: with anything else elsewhere that is an error, not a pointer."""
    import torch
    z = lambda *s, dtype=torch.bfloat16, device="cpu": torch.zeros(s, dtype=dtype, device=device)
    ints = lambda *s, device="cpu": torch.zeros(s, dtype=torch.int32, device=device)
    x, f, at = z(5, 4, 64), torch.ones(16), ints(5)
    for args in ((x, x, f.to("meta"), at), (x, x, f, at.to("meta")), (x, x.to("meta"), f, at), (x.to("meta"), x.to("meta"), f, at)):
        with pytest.raises(AssertionError, match="different devices"):
            B.rope_bf16(*args)
    cache = B.PagedCache.empty(6, 4, 16, 64, device="cpu")
    good = [x, x, ints(3), ints(2), ints(2, 3), cache, f, at]
    B.kv_append_fp8(*good)
    for i in (1, 2, 3, 4, 6, 7):
        with pytest.raises(AssertionError, match="different devices"):
            B.kv_append_fp8(*good[:i], good[i].to("meta"), *good[i + 1:])
    for name in cache._fields:
        with pytest.raises(AssertionError, match="different devices"):
            B.kv_append_fp8(*good[:5], cache._replace(**{name: getattr(cache, name).to("meta")}))
    q, wide = z(2, 8, 64), ints(2, 100)
    room = z(B.attn_paged_scratch_bytes(2, 8, 4, 64, 16, 100), dtype=torch.uint8)
    good = [q, cache, wide, ints(2), z(2, 8, 64), room]
    B.attn_paged_fp8(*good)
    for i in (0, 2, 3, 4, 5):
        with pytest.raises(AssertionError, match="different devices"):
            B.attn_paged_fp8(*good[:i], good[i].to("meta"), *good[i + 1:])


def test_rows_further_apart_than_32_bits_are_refused(B):
    """2^32 elements between tokens, or entries between a table's rows, would be taken for dense ones."""
    import torch
    far = lambda *s, dtype=torch.bfloat16: torch.empty_strided(s, (1 << 32, *(64, 1)[3 - len(s):]), dtype=dtype, device="meta")
    m = lambda *s, dtype=torch.int32: torch.empty(s, dtype=dtype, device="meta")
    x, f = far(5, 4, 64), m(16, dtype=torch.float32)
    near = m(5, 4, 64, dtype=torch.bfloat16)
    for args in ((x, near, f, m(5)), (near, x, f, m(5))):
        with pytest.raises(AssertionError, match="too far"):
            B.rope_bf16(*args)
    cache = B.PagedCache.empty(6, 4, 16, 64, device="meta")
    with pytest.raises(AssertionError, match="too far"):
        B.kv_append_fp8(x, near, m(3), m(2), m(2, 3), cache)
    with pytest.raises(AssertionError, match="too far"):
        B.attn_paged_fp8(m(2, 4, 64, dtype=torch.bfloat16), cache, far(2, 3, dtype=torch.int32), m(2), m(2, 4, 64, dtype=torch.bfloat16))


def test_workers_of_an_append_leave_room_for_others(B, tmp_path):
    """Prompts as workers: 128 registers at most, four waves on a SIMD, and nothing in memory beside them."""
    import re
    from test_host_logic import _device_code
    notes = _device_code(B, tmp_path)("llvm-readelf", "--notes")
    found = {}
    for kernel in notes.split("- .agpr_count:")[1:]:
        get = lambda key: re.search(r"\." + key + r":\s+(\S+)", kernel).group(1)
        if "ptb" in get("name") and re.search(r"AppendBodyTILi\d+ELi\d+ELi0E", get("name")):
            found[get("name")] = (int(get("vgpr_count")) + int(kernel.split()[0]), int(get("private_segment_fixed_size")))
    assert len(found) == 5 and all(r[0] <= 128 and r[1] == 0 for r in found.values()), found
