"""Host-side checks of the entry points of the cache in 4 bits: every invalid
call is refused before any HIP call (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2609_33390_amd as brisk

ENULL, ESHAPE, EUNSUP, EWS = -1, -2, -3, -4
FAKE, ODD = 0x10000, 0x10002       # aligned and misaligned addresses, never dereferenced
PAGES = 0x40000000
BIG = 1 << 60
PART = 64 * 136                    # bytes of a page's part of 64 slots


def _cache(**kw):
    a = dict(dtype=0, n_kv_heads=8, d_head=128, page_size=64, n_pages=100, max_pages=32, page_stride=8 * PART,
             head_stride=PART, pages=PAGES, block_table=FAKE, seq_len=FAKE)
    a.update(kw)
    return brisk._KVCache4C(**a)


BAD_CACHE = [
    (dict(pages=None), ENULL), (dict(block_table=None), ENULL), (dict(seq_len=None), ENULL), (dict(dtype=2), ESHAPE),
    (dict(dtype=-1), ESHAPE), (dict(n_kv_heads=0), ESHAPE), (dict(n_kv_heads=1025), ESHAPE), (dict(d_head=0), ESHAPE),
    (dict(d_head=136), ESHAPE), (dict(d_head=100), EUNSUP), (dict(page_size=8), ESHAPE), (dict(page_size=1 << 17), ESHAPE),
    (dict(page_size=48), EUNSUP), (dict(n_pages=0), ESHAPE), (dict(max_pages=0), ESHAPE), (dict(max_pages=1 << 25), ESHAPE),
    (dict(page_stride=-16), ESHAPE), (dict(head_stride=-16), ESHAPE), (dict(page_stride=8 * PART + 8), EUNSUP),
    (dict(head_stride=PART + 8), EUNSUP), (dict(pages=PAGES + 8), EUNSUP), (dict(block_table=ODD), EUNSUP),
    (dict(seq_len=ODD), EUNSUP),
]


def _write(c=None, **kw):
    a = dict(k=FAKE, v=FAKE, seq=16 * 4096, row=4096, head=128, B=4, T=16, first=FAKE, count=FAKE)
    a.update(kw)
    return brisk.lib().brisk_kv4_write(ctypes.byref(_cache() if c is None else c), a["k"], a["v"], a["seq"], a["row"],
                                       a["head"], a["B"], a["T"], a["first"], a["count"], None)


def _read(c=None, **kw):
    a = dict(B=4, T=16, first=FAKE, k=0x20000000, v=0x30000000)
    a.update(kw)
    return brisk.lib().brisk_kv4_read(ctypes.byref(_cache() if c is None else c), a["B"], a["T"], a["first"], a["k"], a["v"], None)


def _attend(c=None, pre=None, **kw):
    a = dict(q=FAKE, row=4096, head=128, mask=None, B=4, L=16, H=32, most=2048, scale=0.1, out=FAKE, lse=FAKE, ws=FAKE,
             ws_bytes=BIG)
    a.update(kw)
    return brisk.lib().brisk_kv4_attention(
        ctypes.byref(_cache() if c is None else c), None if pre is None else ctypes.byref(pre), a["q"], a["row"],
        a["head"], a["mask"], a["B"], a["L"], a["H"], a["most"], a["scale"], a["out"], a["lse"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,want", BAD_CACHE)
def test_cache_is_checked_by_every_call(kw, want):
    c = _cache(**kw)
    assert _write(c) == want
    assert _read(c) == want
    assert _attend(c) == want


@pytest.mark.parametrize("kw,want", [
    (dict(k=None), ENULL), (dict(v=None), ENULL), (dict(first=None), ENULL), (dict(B=0), ESHAPE), (dict(T=0), ESHAPE),
    (dict(B=-1), ESHAPE), (dict(T=(1 << 30) + 1), ESHAPE), (dict(B=1 << 23), ESHAPE), (dict(T=1 << 29), ESHAPE),
    (dict(seq=-8), ESHAPE), (dict(row=-8), ESHAPE), (dict(head=-8), ESHAPE), (dict(seq=4), EUNSUP), (dict(row=4), EUNSUP),
    (dict(head=4), EUNSUP), (dict(k=ODD), EUNSUP), (dict(v=ODD), EUNSUP), (dict(first=ODD), EUNSUP), (dict(count=ODD), EUNSUP),
    # the pages overlap what the call reads
    (dict(k=PAGES + 4096), EUNSUP), (dict(v=PAGES - 1024), EUNSUP), (dict(first=PAGES), EUNSUP),
    (dict(count=PAGES + 100 * 8 * PART - 4), EUNSUP),
])
def test_write_validation(kw, want):
    assert _write(**kw) == want


@pytest.mark.parametrize("kw", [
    dict(head_stride=PART - 16), dict(head_stride=0), dict(page_stride=8 * PART - 16), dict(page_stride=0),
    dict(head_stride=99 * PART, page_stride=PART), dict(head_stride=100 * PART, page_stride=PART - 16),
    dict(block_table=PAGES), dict(seq_len=PAGES + 16),
])
def test_write_refuses_pages_that_share_memory(kw):
    assert _write(_cache(**kw)) == EUNSUP


@pytest.mark.parametrize("kw,want", [
    (dict(k=None), ENULL), (dict(v=None), ENULL), (dict(B=0), ESHAPE), (dict(T=0), ESHAPE), (dict(T=-3), ESHAPE),
    (dict(T=1 << 29), ESHAPE), (dict(k=ODD), EUNSUP), (dict(v=ODD), EUNSUP), (dict(first=ODD), EUNSUP),
    (dict(k=FAKE), EUNSUP), (dict(v=FAKE), EUNSUP), (dict(v=0x20000000), EUNSUP), (dict(k=PAGES), EUNSUP),
    (dict(v=PAGES + 100 * 8 * PART - 16), EUNSUP), (dict(k=PAGES - 4 * 16 * 8 * 256 + 16), EUNSUP), (dict(v=0x20000000 + 4 * 16 * 8 * 256 - 16), EUNSUP),
])
def test_read_validation(kw, want):
    assert _read(**kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), ENULL), (dict(out=None), ENULL), (dict(B=0), ESHAPE), (dict(L=0), ESHAPE), (dict(L=65), ESHAPE),
    (dict(H=0), ESHAPE), (dict(H=30), ESHAPE), (dict(B=(1 << 13) + 1), ESHAPE), (dict(most=-1), ESHAPE),
    (dict(most=2049), ESHAPE), (dict(scale=0.0), ESHAPE), (dict(scale=-1.0), ESHAPE), (dict(scale=float("nan")), ESHAPE),
    (dict(scale=float("inf")), ESHAPE), (dict(scale=2e30), ESHAPE), (dict(row=-8), ESHAPE), (dict(head=-8), ESHAPE),
    (dict(row=4100), EUNSUP), (dict(head=4), EUNSUP), (dict(q=ODD), EUNSUP), (dict(out=ODD), EUNSUP), (dict(lse=ODD), EUNSUP),
    (dict(mask=0x10004), EUNSUP), (dict(ws=ODD, B=1, L=1), EUNSUP),
])
def test_attention_validation(kw, want):
    assert _attend(**kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(k=None), ENULL), (dict(v=None), ENULL), (dict(len=-1), ESHAPE), (dict(len=(1 << 30) + 1), ESHAPE),
    (dict(slot_stride=-8), ESHAPE), (dict(head_stride=-8), ESHAPE), (dict(slot_stride=4), EUNSUP),
    (dict(head_stride=4), EUNSUP), (dict(k=ODD), EUNSUP), (dict(v=ODD), EUNSUP),
])
def test_prefix_validation(kw, want):
    a = dict(len=100, slot_stride=1024, head_stride=128, k=FAKE, v=FAKE)
    a.update(kw)
    assert _attend(pre=brisk._KVPrefixC(**a)) == want


def test_attention_workspace():
    need = brisk._kv4_workspace_size(1, 1, 32, 8, 128, 1000, 2048)    # prefix and own runs are joined
    assert need > 0
    pre = brisk._KVPrefixC(len=1000, slot_stride=1024, head_stride=128, k=FAKE, v=FAKE)
    assert _attend(pre=pre, B=1, L=1, ws=None, ws_bytes=0) == EWS
    assert _attend(pre=pre, B=1, L=1, ws_bytes=need - 1) == EWS
    L, n = brisk.lib(), ctypes.c_size_t(7)
    assert L.brisk_kv4_attention_workspace_size(1, 1, 32, 8, 128, 0, 100, None) == ENULL
    for bad in ((0, 1, 32, 8, 128, 0, 100), (1, 65, 32, 8, 128, 0, 100), (1, 1, 30, 8, 128, 0, 100), (1, 1, 32, 8, 136, 0, 100),
                (1, 1, 32, 8, 128, -1, 100), (1, 1, 32, 8, 128, 0, -1), (1 << 22, 1, 32, 8, 128, 0, 1)):
        assert L.brisk_kv4_attention_workspace_size(*bad, ctypes.byref(n)) == ESHAPE
    assert n.value == 7


@pytest.mark.parametrize("page,d,want", [(16, 128, 16 * 136), (64, 72, 64 * 136), (16, 64, 16 * 72), (65536, 8, 65536 * 72)])
def test_page_bytes(page, d, want):
    assert brisk.kv4_page_bytes(page, d) == want


@pytest.mark.parametrize("page,d,want", [(8, 128, ESHAPE), (1 << 17, 128, ESHAPE), (48, 128, EUNSUP), (64, 136, ESHAPE),
                                         (64, 0, ESHAPE), (64, 100, EUNSUP)])
def test_page_bytes_refuses(page, d, want):
    with pytest.raises(brisk.BriskError) as e:
        brisk.kv4_page_bytes(page, d)
    assert e.value.status == want
    assert brisk.lib().brisk_kv4_page_bytes(64, 128, None) == ENULL


def test_host_tensors_are_refused():
    pages = torch.zeros(2, 4, brisk.kv4_page_bytes(16, 64), dtype=torch.uint8)
    table, n = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for bad, err in ((pages, ValueError), (pages.float(), TypeError), (None, TypeError), (pages[0], ValueError)):
        with pytest.raises(err):
            brisk.KVCache4(bad, table, n, 64)
    for call in (lambda: brisk.kv4_read(None, 4), lambda: brisk.kv4_write(pages, pages, None, n),
                 lambda: brisk.kv4_attention(pages, None)):
        with pytest.raises(TypeError):
            call()
