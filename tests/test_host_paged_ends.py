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
