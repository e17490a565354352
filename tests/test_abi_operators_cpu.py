"""Host-side checks of the attention, cache and draft entry points: every
invalid call is refused before any HIP call (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2609_33390_amd as brisk

ENULL, ESHAPE, EUNSUP, EWS = -1, -2, -3, -4
FAKE, ODD = 0x10000, 0x10002       # aligned and misaligned addresses, never dereferenced
BIG = 1 << 60


def _cache(**kw):
    a = dict(dtype=0, n_kv_heads=8, d_head=128, page_size=64, n_pages=100, max_pages=32, page_stride=64 * 1024,
             slot_stride=1024, head_stride=128, k_pages=FAKE, v_pages=FAKE, block_table=FAKE, seq_len=FAKE)
    a.update(kw)
    return brisk._KVCacheC(**a)


BAD_CACHE = [
    (dict(k_pages=None), ENULL), (dict(v_pages=None), ENULL), (dict(block_table=None), ENULL), (dict(seq_len=None), ENULL),
    (dict(dtype=2), ESHAPE), (dict(dtype=-1), ESHAPE), (dict(n_kv_heads=0), ESHAPE), (dict(n_kv_heads=1025), ESHAPE),
    (dict(d_head=0), ESHAPE), (dict(d_head=136), ESHAPE), (dict(d_head=100), EUNSUP), (dict(page_size=0), ESHAPE),
    (dict(page_size=1 << 17), ESHAPE), (dict(page_size=48), EUNSUP), (dict(n_pages=0), ESHAPE), (dict(max_pages=0), ESHAPE),
    (dict(max_pages=1 << 25), ESHAPE), (dict(page_stride=-8), ESHAPE), (dict(slot_stride=1020), EUNSUP),
    (dict(head_stride=4), EUNSUP), (dict(page_stride=12), EUNSUP), (dict(k_pages=ODD), EUNSUP), (dict(v_pages=ODD), EUNSUP),
    (dict(block_table=ODD), EUNSUP), (dict(seq_len=ODD), EUNSUP),
]


def _attend(c=None, pre=None, **kw):
    a = dict(q=FAKE, row=4096, head=128, mask=None, B=4, L=16, H=32, most=2048, scale=0.1, out=FAKE, lse=FAKE, ws=FAKE,
             ws_bytes=BIG)
    a.update(kw)
    return brisk.lib().brisk_block_attention(
        ctypes.byref(_cache() if c is None else c), None if pre is None else ctypes.byref(pre), a["q"], a["row"],
        a["head"], a["mask"], a["B"], a["L"], a["H"], a["most"], a["scale"], a["out"], a["lse"], a["ws"], a["ws_bytes"], None)


def _prefix(**kw):
    a = dict(len=100, slot_stride=1024, head_stride=128, k=FAKE, v=FAKE)
    a.update(kw)
    return brisk._KVPrefixC(**a)


@pytest.mark.parametrize("kw,want", BAD_CACHE)
def test_cache_is_checked_by_every_call(kw, want):
    c = _cache(**kw)
    assert _attend(c) == want
    assert _score(c) == want
    assert _evict(c) == want


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), ENULL), (dict(out=None), ENULL), (dict(B=0), ESHAPE), (dict(L=0), ESHAPE), (dict(L=65), ESHAPE),
    (dict(H=0), ESHAPE), (dict(H=30), ESHAPE), (dict(B=1 << 24), ESHAPE), (dict(B=(1 << 15) + 1), ESHAPE), (dict(most=-1), ESHAPE),
    (dict(most=2049), ESHAPE), (dict(scale=0.0), ESHAPE), (dict(scale=-1.0), ESHAPE), (dict(scale=float("nan")), ESHAPE),
    (dict(scale=float("inf")), ESHAPE), (dict(scale=2e30), ESHAPE), (dict(row=-8), ESHAPE), (dict(head=-8), ESHAPE),
    (dict(row=4100), EUNSUP),
    (dict(head=4), EUNSUP), (dict(q=ODD), EUNSUP), (dict(out=ODD), EUNSUP), (dict(lse=ODD), EUNSUP),
    (dict(mask=0x10004), EUNSUP),
])
def test_attention_validation(kw, want):
    assert _attend(**kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(k=None), ENULL), (dict(v=None), ENULL), (dict(len=-1), ESHAPE), (dict(len=(1 << 30) + 1), ESHAPE),
    (dict(slot_stride=-8), ESHAPE), (dict(head_stride=-8), ESHAPE), (dict(slot_stride=4), EUNSUP),
    (dict(head_stride=4), EUNSUP), (dict(k=ODD), EUNSUP), (dict(v=ODD), EUNSUP),
])
def test_prefix_validation(kw, want):
    assert _attend(pre=_prefix(**kw)) == want


def test_attention_workspace():
    n = brisk.block_attention_workspace_size(4, 16, 32, 8, 128, 0, 2048)
    if n:
        assert _attend(ws_bytes=n - 1) == EWS
        assert _attend(ws=None) == EWS
    assert _attend(ws=0x10008) == EUNSUP
    L = brisk.lib()
    assert L.brisk_block_attention_workspace_size(4, 16, 32, 8, 128, 0, 2048, None) == ENULL
    for bad, want in (((0, 16, 32, 8, 128, 0, 64), ESHAPE), ((4, 65, 32, 8, 128, 0, 64), ESHAPE),
                      ((4, 16, 31, 8, 128, 0, 64), ESHAPE), ((4, 16, 32, 8, 256, 0, 64), ESHAPE),
                      ((4, 16, 32, 8, 68, 0, 64), EUNSUP), ((4, 16, 32, 8, 128, -1, 64), ESHAPE),
                      ((4, 16, 32, 8, 128, 0, -1), ESHAPE), ((4, 16, 32, 0, 128, 0, 64), ESHAPE)):
        out = ctypes.c_size_t(77)
        assert L.brisk_block_attention_workspace_size(*bad, ctypes.byref(out)) == want and out.value == 77


def _score(c=None, **kw):
    a = dict(q=FAKE, row=4096, head=128, mask=None, lse=FAKE, B=4, L=16, H=32, scale=0.1, decay=1.0, si=FAKE, so=FAKE, cap=2048)
    a.update(kw)
    return brisk.lib().brisk_cache_score(ctypes.byref(_cache() if c is None else c), a["q"], a["row"], a["head"], a["mask"],
                                         a["lse"], a["B"], a["L"], a["H"], a["scale"], a["decay"], a["si"], a["so"],
                                         a["cap"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), ENULL), (dict(lse=None), ENULL), (dict(si=None), ENULL), (dict(so=None), ENULL), (dict(B=0), ESHAPE),
    (dict(L=65), ESHAPE), (dict(H=12), ESHAPE), (dict(cap=0), ESHAPE), (dict(cap=(1 << 30) + 1), ESHAPE),
    (dict(scale=0.0), ESHAPE), (dict(row=-8), ESHAPE), (dict(q=ODD), EUNSUP), (dict(row=4), EUNSUP), (dict(head=4), EUNSUP),
    (dict(lse=ODD), EUNSUP), (dict(si=ODD), EUNSUP), (dict(so=ODD), EUNSUP), (dict(mask=0x10004), EUNSUP),
])
def test_score_validation(kw, want):
    assert _score(**kw) == want


@pytest.mark.parametrize("kw", [
    dict(so=(1 << 24) + 16), dict(so=(1 << 24) - 16), dict(so=2 << 24), dict(so=(2 << 24) + 4 * 16 * 32 * 4 - 4),
    dict(so=3 << 24), dict(so=4 << 24), dict(so=5 << 24),
])
def test_score_refuses_overlapping_buffers(kw):
    """The whole array may be updated in place, but not one shifted against itself."""
    apart = dict(si=1 << 24, lse=2 << 24, mask=5 << 24)
    assert _score(_cache(seq_len=3 << 24, block_table=4 << 24), **{**apart, **kw}) == EUNSUP


def _evict(c=None, **kw):
    a = dict(B=4, si=FAKE, pi=FAKE, cap=2048, np_=FAKE, budget=512, recent=16, so=FAKE, po=FAKE, nl=FAKE, ws=FAKE, ws_bytes=BIG)
    a.update(kw)
    return brisk.lib().brisk_cache_evict(ctypes.byref(_cache() if c is None else c), a["B"], a["si"], a["pi"], a["cap"],
                                         a["np_"], a["budget"], a["recent"], a["so"], a["po"], a["nl"], a["ws"],
                                         a["ws_bytes"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(si=None), ENULL), (dict(pi=None), ENULL), (dict(np_=None), ENULL), (dict(so=None), ENULL), (dict(po=None), ENULL),
    (dict(nl=None), ENULL), (dict(B=0), ESHAPE), (dict(B=1 << 20), ESHAPE), (dict(cap=0), ESHAPE),
    (dict(cap=(1 << 24) + 1), ESHAPE), (dict(budget=0), ESHAPE), (dict(recent=-1), ESHAPE), (dict(recent=513), ESHAPE),
    (dict(si=ODD), EUNSUP), (dict(pi=ODD), EUNSUP), (dict(np_=ODD), EUNSUP), (dict(so=ODD), EUNSUP), (dict(po=ODD), EUNSUP),
    (dict(nl=ODD), EUNSUP), (dict(ws_bytes=8), EWS), (dict(ws=None), EWS), (dict(ws=0x10008), EUNSUP),
])
def test_evict_validation(kw, want):
    assert _evict(**kw) == want


SLOTS = 4 * 8 * 2048 * 4            # bytes of a score or position array of _evict's sizes
APART = dict(si=1 << 24, pi=2 << 24, np_=3 << 24, so=4 << 24, po=5 << 24, nl=6 << 24, ws=7 << 24, ws_bytes=1 << 24)
LENS, TABLE = 8 << 24, 9 << 24


@pytest.mark.parametrize("kw", [
    dict(nl=LENS), dict(nl=LENS + 12), dict(nl=LENS - 12), dict(nl=APART["np_"]), dict(nl=TABLE + 4 * 32 * 4 - 4),
    dict(nl=APART["si"] + SLOTS - 4), dict(nl=APART["so"] + 8), dict(nl=APART["ws"]), dict(so=APART["si"]),
    dict(so=APART["si"] + SLOTS - 16), dict(so=APART["pi"] - 16), dict(po=APART["si"]), dict(po=APART["pi"] + 16),
    dict(po=APART["so"]), dict(ws=APART["si"]), dict(ws=APART["pi"] + 16), dict(ws=LENS), dict(ws=TABLE), dict(ws=APART["po"]),
])
def test_evict_refuses_overlapping_buffers(kw):
    """Lengths cut in place among them: later launches would take lists that nobody wrote."""
    assert _evict(_cache(seq_len=LENS, block_table=TABLE), **{**APART, **kw}) == EUNSUP


@pytest.mark.parametrize("kw,bad", [
    (dict(head_stride=0), True), (dict(slot_stride=0), True), (dict(page_stride=0), True),       # expanded dimensions
    (dict(head_stride=120), True), (dict(slot_stride=1016), True), (dict(page_stride=64 * 1024 - 8), True),
    (dict(page_stride=64 * 1024, slot_stride=128, head_stride=64 * 128), False),                  # head-major pages
    (dict(page_stride=128, slot_stride=12800, head_stride=64 * 12800), False),                    # pages innermost
    (dict(n_kv_heads=1, head_stride=0), False), (dict(page_size=1, slot_stride=0), False),
    (dict(n_pages=1, page_stride=0), False), (dict(page_stride=1 << 62), False),
])
def test_evict_refuses_pages_that_share_memory(kw, bad):
    """Where two heads are one in memory each would move rows under the other; reading them is fine."""
    assert _evict(_cache(**kw), ws_bytes=0) == (EUNSUP if bad else EWS)


def test_calls_that_no_launch_holds_are_refused():
    """2^32 threads or more: refused as a shape, before anything is launched."""
    one = dict(n_kv_heads=1, max_pages=1 << 14, page_size=1 << 16)
    assert _score(_cache(**one), B=1 << 24, L=1, H=1, cap=1) == ESHAPE
    assert _score(_cache(**one), B=1 << 14, L=1, H=1, cap=1 << 20) == ESHAPE
    assert _score(_cache(**one), B=1 << 16, L=1, H=1, cap=1 << 20) == ESHAPE
    size = brisk.lib().brisk_cache_evict_workspace_size
    for B, Hkv, cap, budget, want in ((1 << 10, 8, 1 << 21, 1 << 20, ESHAPE), (1 << 10, 8, 1 << 18, 1 << 17, ESHAPE),
                                      (1 << 10, 8, (1 << 18) - 128, 1 << 16, 0), (1 << 10, 8, 1 << 21, 1000, 0),
                                      (1 << 20, 1, 33000, 1, ESHAPE), (1 << 18, 1, 33000, 1, 0)):
        n = ctypes.c_size_t(77)
        assert size(B, Hkv, cap, budget, ctypes.byref(n)) == want, (B, Hkv, cap, budget)
        assert (n.value == 77) == (want != 0)
        if want:
            assert _evict(_cache(n_kv_heads=Hkv), B=B, cap=cap, budget=budget, **{k: APART[k] for k in APART}) == want


def test_attention_splits_no_finer_than_a_launch_holds():
    """Millions of workgroups are not split further, however long their caches may be."""
    most = (1 << 23) + 1                            # whole caches: one run of each row, no workspace
    assert brisk.block_attention_workspace_size(most, 1, 1, 1, 8, 0, 1 << 30) == 0


def _draft(**kw):
    a = dict(t=FAKE, ts=1000, d=FAKE, ds=1000, tok=FAKE, n=None, u=FAKE, e=FAKE, es=1000, B=4, L=8, V=1000, acc=FAKE,
             out=FAKE, ws=FAKE, ws_bytes=BIG)
    a.update(kw)
    return brisk.lib().brisk_draft_verify(a["t"], a["ts"], a["d"], a["ds"], a["tok"], a["n"], a["u"], a["e"], a["es"], a["B"],
                                          a["L"], a["V"], a["acc"], a["out"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(t=None), ENULL), (dict(d=None), ENULL), (dict(tok=None), ENULL), (dict(u=None), ENULL), (dict(e=None), ENULL),
    (dict(acc=None), ENULL), (dict(out=None), ENULL), (dict(B=0), ESHAPE), (dict(L=-1), ESHAPE), (dict(L=1025), ESHAPE),
    (dict(V=0), ESHAPE), (dict(V=(1 << 24) + 1, ts=BIG, ds=BIG, es=BIG), ESHAPE), (dict(ts=999), ESHAPE),
    (dict(ds=999), ESHAPE), (dict(es=999), ESHAPE), (dict(B=1 << 19), ESHAPE), (dict(t=ODD), EUNSUP), (dict(d=ODD), EUNSUP),
    (dict(tok=ODD), EUNSUP), (dict(n=ODD), EUNSUP), (dict(u=ODD), EUNSUP), (dict(e=ODD), EUNSUP), (dict(acc=ODD), EUNSUP),
    (dict(out=ODD), EUNSUP), (dict(ws=0x10008), EUNSUP),
])
def test_draft_validation(kw, want):
    assert _draft(**kw) == want


def test_binding_refuses_host_tensors_and_wrong_types():
    k = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        brisk.KVCache(k, k, torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(TypeError):
        brisk.KVCache(k.float(), k.float(), torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(TypeError):
        brisk.KVCache(None, k, None, None)
    p = torch.zeros(1, 3, 7)
    with pytest.raises(ValueError):
        brisk.draft_verify(p, p[:, :2], torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, 2), torch.zeros(1, 7))
