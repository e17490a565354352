"""GPU checks of brisk_cache_score and brisk_cache_evict against the float64 oracle.

A score's terms exp(s - lse) carry the rounding of a 32-bit logit (2^-19 of
scale * sum |q k|), of the subtraction and of the exponential; with the sum of
at most 64 x 16 of them each result stays within 2^-18 of the oracle's error
scale sum p (2 + |lse| + scale sum |q k|).  Eviction moves values: exact."""
import numpy as np
import pytest
import torch

import oracle.attention_oracle as ao
from kv_cases import Case

pytestmark = pytest.mark.gpu

brisk = pytest.importorskip("paper_2609_33390_amd")


SCORE_CASES = [
    dict(B=1, L=1, H=4, Hkv=4, D=128, lens=[1]),
    dict(B=4, L=1, H=8, Hkv=2, D=128, lens=[0, 1, 33, 300], page=1),
    dict(B=3, L=16, H=8, Hkv=2, D=128, lens=[3, 17, 260], mask="mixed", page=64),
    dict(B=2, L=33, H=6, Hkv=6, D=80, lens=[33, 130], mask="random", layout="hnd", dtype="f16"),
    dict(B=2, L=64, H=16, Hkv=1, D=64, lens=[64, 150], mask="causal"),
    dict(B=2, L=7, H=4, Hkv=4, D=8, lens=[7, 5], mask="hidden"),
    dict(B=2, L=5, H=15, Hkv=5, D=104, lens=[129, 31], mask="causal", page=8),
    dict(B=1, L=2, H=14, Hkv=2, D=128, lens=[5000], mask="causal", page=128),
    dict(B=2, L=40, H=7, Hkv=1, D=96, lens=[400, 41], mask="mixed", dtype="f16"),
    # enough heads for long runs of tiles, with more rows than a wavefront holds
    dict(B=66, L=5, H=128, Hkv=8, D=16, lens=[3 * b for b in range(66)], mask="causal"),
]


def _score_inputs(c, extra_cap):
    own_k = c.own(c.k)
    _, lse, _, _ = ao.block_attention(c.q.double().numpy(), own_k, c.own(c.v), None, c.mask, c.scale)
    lse = (lse + 0.25).astype(np.float32)          # part of the weight lies elsewhere
    cap = max(1, max(c.lens)) + extra_cap
    score = c.rng.random((c.B, c.Hkv, cap)).astype(np.float32)
    return own_k, lse, score


@pytest.mark.parametrize("kw", SCORE_CASES)
def test_score_matches_oracle(kw):
    c = Case(prefix=None, seed=len(str(kw)), **kw)
    print(f"[score] {kw}", flush=True)
    own_k, lse, score = _score_inputs(c, 37)
    want, err = ao.cache_score(c.q.double().numpy(), own_k, lse.astype(np.float64), c.mask, c.scale, 0.75, score)
    args = (c.q.cuda(), torch.from_numpy(lse).cuda(), c.cache(brisk))
    s = torch.from_numpy(score).cuda()
    got = brisk.cache_score(*args, s, block_mask=c.gpu_mask(), scale=c.scale, decay=0.75)
    again = brisk.cache_score(*args, s, block_mask=c.gpu_mask(), scale=c.scale, decay=0.75, out=s)   # in place
    torch.cuda.synchronize()
    assert again is s and torch.equal(got, again)
    assert (np.abs(got.double().cpu().numpy() - want) <= 2.0 ** -18 * err).all()


def test_score_is_cut_to_its_capacity():
    c = Case(2, 4, 4, 2, 64, None, [200, 30], mask="causal", seed=3)
    own_k, lse, score = _score_inputs(c, 0)
    cap = 77
    c.lens = [77, 30]                              # a sequence longer than the scores: its first 77 slots
    cut = [k[:n] for k, n in zip(own_k, c.lens)]
    want, err = ao.cache_score(c.q.double().numpy(), cut, lse.astype(np.float64), c.mask, c.scale, 1.0, score[:, :, :cap])
    cache = c.cache(brisk)
    cache.seq_len.copy_(torch.tensor([200, 30], dtype=torch.int32))
    got = brisk.cache_score(c.q.cuda(), torch.from_numpy(lse).cuda(), cache,
                            torch.from_numpy(score[:, :, :cap].copy()).cuda(), block_mask=c.gpu_mask(), scale=c.scale)
    assert (np.abs(got.double().cpu().numpy() - want) <= 2.0 ** -18 * err).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_score_ignores_hidden_keys(bad):
    """A key no row sees gets nothing, whatever it holds; its neighbours are unaffected."""
    c = Case(2, 8, 8, 2, 128, None, [100, 40], mask="hidden", seed=4)
    own_k, lse, score = _score_inputs(c, 5)
    want, err = ao.cache_score(c.q.double().numpy(), own_k, lse.astype(np.float64), c.mask, c.scale, 1.0, score)
    for b, n in enumerate(c.lens):
        for j in (n - 1, n - 8):
            c.k[c.table[b, j // c.page], j % c.page] = bad
    got = brisk.cache_score(c.q.cuda(), torch.from_numpy(lse).cuda(), c.cache(brisk), torch.from_numpy(score).cuda(),
                            block_mask=c.gpu_mask(), scale=c.scale).double().cpu().numpy()
    assert (np.abs(got - want) <= 2.0 ** -18 * err).all()


def test_scores_sum_to_the_rows_weight():
    """With the lse of block_attention over the same keys every row spreads a weight of one."""
    c = Case(3, 8, 16, 4, 128, None, [500, 64, 9], mask="causal", seed=5)
    cache, q, mask = c.cache(brisk), c.q.cuda(), c.gpu_mask()
    _, lse = brisk.block_attention(q, cache, block_mask=mask)
    s = brisk.cache_score(q, lse, cache, torch.zeros(3, 4, 500, device="cuda"), block_mask=mask)
    total = s.double().sum(-1).cpu().numpy()       # 8 positions x 4 query heads of each group
    assert np.abs(total - 32.0).max() <= 32 * 2.0 ** -16


def test_score_stays_inside_and_repeats():
    from test_gpu_canary import Guarded
    c = Case(2, 16, 8, 2, 128, None, [130, 77], mask="mixed", seed=6)
    _, lse, score = _score_inputs(c, 3)
    out = Guarded(score.shape, torch.float32)
    cache, s, z = c.cache(brisk), torch.from_numpy(score).cuda(), torch.from_numpy(lse).cuda()
    a = brisk.cache_score(c.q.cuda(), z, cache, s, block_mask=c.gpu_mask(), out=out.t).clone()
    assert out.intact()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        b = brisk.cache_score(c.q.cuda(), z, cache, s, block_mask=c.gpu_mask())
    torch.cuda.synchronize()
    assert torch.equal(a, b)


# ------------------------------------------------------------------- eviction
class EvictCase:
    def __init__(self, lens, budget, recent, Hkv=2, D=64, page=16, layout="nhd", dtype="bf16", extra=5, seed=0, kind="mass"):
        B = len(lens)
        self.c = Case(B, 1, Hkv, Hkv, D, None, lens, page=page, layout=layout, dtype=dtype, seed=seed, junk=0.0)
        rng = self.c.rng
        self.cap = max(1, max(lens)) + extra
        shape = (B, Hkv, self.cap)
        self.budget, self.recent = budget, recent
        if kind == "mass":
            self.score = np.exp(1.5 * rng.standard_normal(shape)).astype(np.float32)
            self.score[rng.random(shape) < 0.1] = 0.0
        elif kind == "ties":
            self.score = rng.integers(0, 3, shape).astype(np.float32)
            self.score[rng.random(shape) < 0.2] *= -0.0
        elif kind == "equal":
            self.score = np.full(shape, 0.25, dtype=np.float32)
        else:                                      # every kind of number
            words = rng.integers(0, 1 << 32, shape, dtype=np.uint64).astype(np.uint32)
            words[rng.random(shape) < 0.1] = 0x7F800000
            words[rng.random(shape) < 0.1] = 0xFF800000
            self.score = words.view(np.float32)
        self.pos = np.stack([np.stack([rng.permutation(self.cap + 9)[:self.cap] for _ in range(Hkv)]) for _ in range(B)])
        self.pos = self.pos.astype(np.int32)
        self.next_pos = np.array([self.cap + 9 if n else 0 for n in lens], dtype=np.int32)

    def want(self):
        c = self.c
        score, pos = np.zeros_like(self.score), np.zeros_like(self.pos)
        k, v = c.k.clone(), c.v.clone()
        for b, n in enumerate(c.lens):
            for h in range(c.Hkv):
                score[b, h], pos[b, h], moves = ao.cache_evict(self.score[b, h], self.pos[b, h], min(n, self.cap),
                                                               self.next_pos[b], self.budget, self.recent)
                for s, d in moves:
                    for x, src in ((k, c.k), (v, c.v)):
                        x[c.table[b, d // c.page], d % c.page, h] = src[c.table[b, s // c.page], s % c.page, h]
        return score, pos, np.minimum(np.minimum(c.lens, self.cap), self.budget), k, v

    def run(self, cache=None, **kw):
        cache = cache or self.c.cache(brisk)
        t = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
        return cache, brisk.cache_evict(cache, t(self.score), t(self.pos), t(self.next_pos), self.budget, self.recent, **kw)


def _same(a, b):
    """Equal bit for bit (every NaN as it came)."""
    return np.array_equal(a.cpu().numpy().view(np.int32), b.view(np.int32))


def _check_evict(e, cache, got):
    score, pos, n, k, v = e.want()
    torch.cuda.synchronize()
    assert np.array_equal(got[2].cpu().numpy(), n)
    assert _same(got[1], pos) and _same(got[0], score)
    assert torch.equal(cache.k_pages.cpu().contiguous().view(torch.int16), k.view(torch.int16))
    assert torch.equal(cache.v_pages.cpu().contiguous().view(torch.int16), v.view(torch.int16))


@pytest.mark.parametrize("kw", [
    dict(lens=[40], budget=17, recent=4),
    dict(lens=[0, 1, 16, 17, 18, 200], budget=17, recent=0),
    dict(lens=[100, 99, 64], budget=64, recent=64, kind="ties"),
    dict(lens=[130, 257], budget=1, recent=1, page=1),
    dict(lens=[130, 257], budget=1, recent=0, kind="equal"),
    dict(lens=[300, 20], budget=299, recent=10, D=128, layout="hnd", dtype="f16"),
    dict(lens=[1000, 700, 2], budget=333, recent=50, Hkv=3, D=80, kind="ties", page=64),
    dict(lens=[513, 1025], budget=512, recent=20, D=8, kind="any"),
    dict(lens=[2049], budget=700, recent=100, Hkv=1, kind="any", layout="hnd"),
    dict(lens=[50, 60], budget=500, recent=3),
    dict(lens=[5000, 4097, 4096], budget=1024, recent=128, Hkv=1, D=16, page=128),
    dict(lens=[70], budget=40, recent=5, extra=-20),            # scores for fewer slots than the sequence holds
])
def test_evict_matches_oracle(kw):
    print(f"[evict] {kw}", flush=True)
    e = EvictCase(seed=len(str(kw)), **kw)
    _check_evict(e, *e.run())


@pytest.mark.parametrize("n,budget,kind", [(20000, 5000, "mass"), (70001, 30000, "ties"), (140000, 1000, "any"),
                                           (40000, 39999, "equal"), (32700, 16000, "any"), (32764, 32000, "ties")])
def test_evict_long_caches(n, budget, kind):
    """Lengths past what one workgroup holds on chip; the oracle's choice by one stable sort."""
    e = EvictCase([n], budget, budget // 8, Hkv=1, D=8, kind=kind, seed=n)
    c = e.c
    print(f"[evict] n={n} budget={budget} {kind}", flush=True)
    score, pos = e.score[0, 0], e.pos[0, 0]
    key = np.where(np.isnan(score[:n]), -np.inf, score[:n].astype(np.float64))
    order = np.where(pos[:n] >= e.next_pos[0] - e.recent, 0, np.where(np.isnan(score[:n]), 2, 1))
    rank = np.lexsort((np.arange(n), np.where(order == 1, -key, 0.0), order))
    kept = np.zeros(n, dtype=bool)
    kept[rank[:budget]] = True
    src, dst = np.nonzero(kept[budget:])[0] + budget, np.nonzero(~kept[:budget])[0]
    ws, wp = np.zeros_like(score), np.full_like(pos, -1)
    ws[:budget], wp[:budget] = score[:budget], pos[:budget]
    ws[dst], wp[dst] = score[src], pos[src]
    cache, got = e.run()
    torch.cuda.synchronize()
    assert _same(got[0], ws[None, None]) and _same(got[1], wp[None, None])
    flat = lambda x: x[torch.from_numpy(c.table[0]).long()].reshape(-1, 8)  # noqa: E731
    for x, y in ((c.k, cache.k_pages), (c.v, cache.v_pages)):
        want = flat(x).clone()
        want[dst] = flat(x)[src]
        assert torch.equal(flat(y.cpu()).view(torch.int16)[:n], want.view(torch.int16)[:n])


@pytest.mark.parametrize("kw", [
    # long, shorter than a chunk, all kept, empty: heads of each over scratch that holds anything
    dict(lens=[40000, 33, 5000, 0], budget=4500, recent=100, Hkv=3, kind="ties", extra=3),
    dict(lens=[700, 33500, 20000], budget=20000, recent=0, Hkv=2, kind="any", layout="hnd", dtype="f16"),
    dict(lens=[32769, 32769, 8193], budget=8192, recent=8192, Hkv=2, kind="mass", page=64),
    dict(lens=[34000, 36864, 12288], budget=1, recent=1, Hkv=4, kind="equal"),
])
def test_evict_batches_of_long_caches(kw):
    """The passes over long caches with several heads and sequences, some of which keep all."""
    import ctypes
    e = EvictCase(D=8, seed=len(str(kw)), **kw)
    c = e.c
    n = ctypes.c_size_t()
    assert e.cap > 32768
    assert brisk.lib().brisk_cache_evict_workspace_size(c.B, c.Hkv, e.cap, e.budget, ctypes.byref(n)) == 0
    ws = torch.full((n.value,), 0xFF, dtype=torch.uint8, device="cuda")
    print(f"[evict] {kw}", flush=True)
    cache, got = e.run(workspace=ws)
    _check_evict(e, cache, got)


def test_evict_twice_and_inside_its_buffers():
    """The inputs stay as they are, so a second call gives the same; nothing outside the buffers is written."""
    from test_gpu_canary import Guarded
    e = EvictCase([300, 90, 41], 64, 9, Hkv=4, seed=21)
    shape = e.score.shape
    so, po, nl = Guarded(shape, torch.float32), Guarded(shape, torch.int32), Guarded((3,), torch.int32)
    import ctypes
    nbytes = ctypes.c_size_t()
    assert brisk.lib().brisk_cache_evict_workspace_size(3, 4, e.cap, 64, ctypes.byref(nbytes)) == 0
    ws = Guarded((nbytes.value,), torch.uint8)
    cache, got = e.run(score_out=so.t, pos_out=po.t, new_len=nl.t, workspace=ws.t)
    _check_evict(e, cache, got)
    assert so.intact() and po.intact() and nl.intact() and ws.intact()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        _, again = e.run(cache)
    torch.cuda.synchronize()
    _check_evict(e, cache, again)


def test_attention_over_an_evicted_cache():
    """After eviction the block attends to what was kept, in whatever order it lies."""
    e = EvictCase([200, 80], 50, 8, Hkv=2, D=64, seed=22)
    c = e.c
    own_k, own_v = c.own(c.k), c.own(c.v)
    cache, (score, pos, n) = e.run()
    cache.seq_len.copy_(n)
    out, _ = brisk.block_attention(c.q.cuda(), cache)
    for b in range(2):
        for h in range(2):
            by_pos = {int(p): j for j, p in enumerate(e.pos[b, h][:c.lens[b]])}
            keep = [by_pos[int(p)] for p in pos[b, h][:50].cpu()]
            s = c.scale * (own_k[b][keep, h] @ c.q[b, 0, h].double().numpy())
            p = np.exp(s - s.max())
            want = p @ own_v[b][keep, h] / p.sum()
            tol = 2.0 ** -8 * (np.abs(want) + p @ np.abs(own_v[b][keep, h]) / p.sum()) + 1e-3
            assert (np.abs(out[b, 0, h].double().cpu().numpy() - want) <= tol).all()


def test_binding_refuses_overlap_and_misfits():
    e = EvictCase([40, 30], 10, 2, seed=23)
    cache = e.c.cache(brisk)
    s, p, n = (torch.from_numpy(x).cuda() for x in (e.score, e.pos, e.next_pos))
    for kw in (dict(score_out=s), dict(pos_out=p), dict(score_out=s[:, :, :-1]), dict(new_len=n[:1]),
               dict(workspace=torch.empty(4, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(ValueError):
            brisk.cache_evict(cache, s, p, n, 10, 2, **kw)
    with pytest.raises(TypeError):
        brisk.cache_evict(cache, s, p.long(), n, 10, 2)
    for budget, recent in ((0, 0), (10, 11), (10, -1)):
        with pytest.raises(brisk.BriskError):
            brisk.cache_evict(cache, s, p, n, budget, recent)
    q, lse = e.c.q.cuda(), torch.zeros(2, 1, 2, device="cuda")
    with pytest.raises(ValueError):
        brisk.cache_score(q, lse[:1], cache, s)
    with pytest.raises(ValueError):
        brisk.cache_score(q, lse, cache, s[:1])
    with pytest.raises(TypeError):
        brisk.cache_score(q, lse, cache, s.double())


def test_binding_refuses_lengths_cut_in_place():
    e = EvictCase([40, 30], 10, 2, seed=24)
    cache = e.c.cache(brisk)
    s, p, n = (torch.from_numpy(x).cuda() for x in (e.score, e.pos, e.next_pos))
    both = torch.zeros(3, dtype=torch.int32, device="cuda")
    shifted = brisk.KVCache(cache.k_pages, cache.v_pages, cache.block_table, both[:2])
    for c, at, out in ((cache, n, cache.seq_len), (cache, n, n), (shifted, n, both[1:]), (shifted, both[1:], both[1:])):
        with pytest.raises(ValueError, match="new_len"):
            brisk.cache_evict(c, s, p, at, 10, 2, new_len=out)
    with pytest.raises(brisk.BriskError) as err:                # and whatever else shares memory, by the library
        brisk.cache_evict(cache, s, p, n, 10, 2, score_out=p.view(torch.float32))
    assert err.value.status == -3


def test_evict_refuses_expanded_heads():
    """Two heads that are one in memory: each would move rows under the other."""
    e = EvictCase([40, 30], 10, 2, seed=25)
    one = e.c.cache(brisk)
    k, v = (x[:, :, :1].expand(-1, -1, 2, -1) for x in (one.k_pages, one.v_pages))
    before = k.clone()
    with pytest.raises(brisk.BriskError) as err:
        e.run(brisk.KVCache(k, v, one.block_table, one.seq_len))
    assert err.value.status == -3
    torch.cuda.synchronize()
    assert torch.equal(k.clone().view(torch.int16), before.view(torch.int16))


def test_a_cache_keeps_its_tensors():
    """Lengths assigned instead of copied would not reach the library: refused."""
    e = EvictCase([40, 30], 10, 2, seed=26)
    cache, (_, _, n) = e.run()
    old = cache.seq_len
    for name in ("seq_len", "k_pages", "v_pages", "block_table"):
        with pytest.raises(AttributeError, match=name):
            setattr(cache, name, n)
    assert cache.seq_len is old and cache.c_struct.seq_len == old.data_ptr()
    old.copy_(n)
    assert cache.seq_len.tolist() == [10, 10]
