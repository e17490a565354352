"""Host-side checks of what a launch on the 4-bit cache holds, at sizes whose product passes
64 bits (no GPU needed)."""
import pytest

from test_abi_kv4_cpu import ESHAPE, PART, _cache, _read, _write

PAST_64_BITS = [
    (1 << 30, 16 * (1 << 24) - 30),                # 2^30 sequences x 1024 heads x 2^24 blocks: 0 in 64 bits
    (1 << 30, 16 * (1 << 24) - 14),                # and one block more of each: 2^40, past the limit all the same
    (1 << 29, 16 * (1 << 25) - 30),
    ((1 << 31) - 1, 1 << 30),
]


@pytest.mark.parametrize("B,T", PAST_64_BITS)
def test_sizes_past_64_bits_are_refused(B, T):
    c = _cache(n_kv_heads=1024, page_stride=1024 * PART, n_pages=1)
    assert _write(c, B=B, T=T, seq=0, row=0, head=0, k=0x10000, v=0x10000) == ESHAPE
    assert _read(c, B=B, T=T) == ESHAPE


@pytest.mark.parametrize("B,Hkv,T,held", [(1 << 15, 1024, 1, False), ((1 << 15) - 1, 1024, 1, True), (1 << 14, 1024, 2, False), ((1 << 14) - 1, 1024, 17, True),
                                          (1, 1, 16 * (1 << 25) - 30, False), (1, 1, 16 * (1 << 25) - 31, True)])
def test_the_limit_itself(B, Hkv, T, held):
    """B * n_kv_heads * ((T + 30) / 16) < 2^25; past it comes the next check, which these outputs fail."""
    c = _cache(n_kv_heads=Hkv, page_stride=Hkv * PART)
    assert (_read(c, B=B, T=T, k=0x20000000, v=0x20000000) == ESHAPE) == (not held)
