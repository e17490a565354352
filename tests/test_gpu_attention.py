"""GPU checks of brisk_block_attention against the float64 oracle.

Tolerances.  With u the unit roundoff of the cache's type, the output's own
rounding gives at most u |out|, and the rounding of each probability where it
meets the values at most u * sum p |v|; 2 * 2^-16 of the same sums covers the
fp32 exponentials, sums and rescaling.  A logit's fp32 sum of D products is
off by less than 2^-19 of scale * sum |q k|, which moves every probability by
that factor and the log-sum-exp by that amount."""
import numpy as np
import pytest
import torch

import oracle.attention_oracle as ao
from kv_cases import TYPES, UNIT, Case

pytestmark = pytest.mark.gpu

brisk = pytest.importorskip("paper_2609_33390_amd")


def _check(c, out, lse, ref=None):
    o, z, mag, size = ref or c.attention()
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    empty = z == -np.inf
    assert np.array_equal(lse == -np.inf, empty)
    assert (out[empty] == 0).all()
    logit = 2.0 ** -19 * size
    tol = UNIT[c.dtype] * (np.abs(o) + mag) + (2.0 ** -15 + 2 * logit[..., None]) * mag + 2.0 ** -24
    assert (np.abs(out - o) <= tol).all(), np.max(np.abs(out - o) / tol)
    assert (np.abs(lse - z)[~empty] <= (logit + 2.0 ** -20 * (1 + np.abs(z)))[~empty]).all()


def _run(c, **kw):
    print(f"[attention] B={c.B} L={c.L} H={c.H}/{c.Hkv} D={c.D} page={c.page} lens={c.lens[:8]} "
          f"prefix={None if c.prefix is None else len(c.prefix[0])} {c.dtype} {c.layout}", flush=True)
    out, lse = brisk.block_attention(c.q.cuda(), c.cache(brisk), prefix=c.gpu_prefix(), block_mask=c.gpu_mask(),
                                     scale=c.scale, **kw)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("kw", [
    # single tokens: lengths of none, one and many, with and without a prefix
    dict(B=1, L=1, H=4, Hkv=4, D=128, prefix=None, lens=[1]),
    dict(B=3, L=1, H=8, Hkv=2, D=128, prefix=None, lens=[0, 1, 300]),
    dict(B=3, L=1, H=8, Hkv=2, D=128, prefix=0, lens=[0, 0, 0]),
    dict(B=5, L=1, H=28, Hkv=4, D=128, prefix=129, lens=[0, 1, 31, 32, 33], page=1),
    dict(B=2, L=1, H=16, Hkv=1, D=64, prefix=1, lens=[65, 2000], page=128, dtype="f16"),
    # blocks: shorter than the block, ending inside tiles and pages
    dict(B=4, L=16, H=8, Hkv=2, D=128, prefix=None, lens=[3, 16, 17, 95], mask="causal"),
    dict(B=3, L=16, H=8, Hkv=2, D=128, prefix=77, lens=[0, 15, 257], mask="mixed", page=64),
    dict(B=2, L=33, H=6, Hkv=6, D=80, prefix=64, lens=[33, 130], mask="random", page=8, layout="hnd"),
    dict(B=2, L=64, H=4, Hkv=2, D=96, prefix=63, lens=[64, 200], mask="random", dtype="f16", layout="hnd"),
    dict(B=1, L=64, H=8, Hkv=1, D=128, prefix=200, lens=[700], mask="mixed"),
    # rows that see nothing
    dict(B=2, L=7, H=4, Hkv=4, D=64, prefix=None, lens=[7, 5], mask="hidden"),
    dict(B=2, L=7, H=4, Hkv=4, D=64, prefix=None, lens=[9, 7], mask="hidden", dtype="f16"),
    # narrow and odd heads
    dict(B=2, L=5, H=3, Hkv=1, D=8, prefix=20, lens=[40, 11], mask="causal"),
    dict(B=2, L=3, H=10, Hkv=5, D=24, prefix=33, lens=[40, 129], mask="causal", dtype="f16"),
    dict(B=1, L=20, H=14, Hkv=2, D=104, prefix=None, lens=[400], mask="causal", page=32),
    dict(B=2, L=4, H=4, Hkv=2, D=72, prefix=300, lens=[100, 50], layout="hnd"),
    # many rows on the prefix
    dict(B=20, L=8, H=8, Hkv=2, D=128, prefix=500, lens=[8 + 7 * b for b in range(20)], mask="mixed", page=32),
    dict(B=70, L=1, H=16, Hkv=2, D=64, prefix=130, lens=[b % 5 for b in range(70)], dtype="f16"),
    dict(B=9, L=31, H=7, Hkv=1, D=128, prefix=193, lens=[31 + 11 * b for b in range(9)], mask="causal"),
    # long caches of few rows, split and joined
    dict(B=1, L=1, H=8, Hkv=8, D=128, prefix=None, lens=[9001], page=64),
    dict(B=2, L=8, H=8, Hkv=2, D=64, prefix=5000, lens=[6000, 37], mask="causal", page=256),
])
def test_attention_matches_oracle(kw):
    c = Case(seed=len(str(kw)), **kw)
    _check(c, *_run(c))


@pytest.mark.parametrize("D", [64, 72, 88, 96, 120, 128])
@pytest.mark.parametrize("kw", [
    dict(B=1, L=1, H=2, Hkv=2, prefix=64, lens=[128]),                       # each row count's tile
    dict(B=2, L=8, H=12, Hkv=2, prefix=128, lens=[64, 192], mask="causal"),
    dict(B=2, L=30, H=6, Hkv=2, prefix=256, lens=[64, 128], mask="mixed"),
    dict(B=4, L=64, H=8, Hkv=2, prefix=192, lens=[64, 64, 128, 320], mask="causal"),
])
def test_full_tiles_up_to_the_end_of_the_pool(D, kw):
    """Whole tiles of keys, the last of them the last of its tensor, for heads that fill their rows of LDS or do not."""
    for dtype in ("bf16", "f16"):
        c = Case(D=D, dtype=dtype, seed=D, page=64, spare_pages=0, **kw)
        _check(c, *_run(c))


@pytest.mark.parametrize("std", [0.0, 30.0])
def test_flat_and_very_sharp_weights(std):
    """All logits equal, and logits of several hundred."""
    c = Case(2, 8, 8, 2, 128, 90, [60, 200], mask="causal", q_std=std, seed=5)
    _check(c, *_run(c))


def test_largest_magnitudes():
    """Values at the type's largest finite number, and keys at its lowest."""
    c = Case(2, 4, 4, 4, 64, None, [40, 9], seed=6, q_std=1e-3)
    top = torch.finfo(torch.bfloat16).max
    c.v[~c.v.isnan()] = top / 256                   # 40 of them still sum below fp32's largest
    out, lse = _run(c)
    assert torch.isfinite(out).all()
    c = Case(1, 2, 2, 2, 64, None, [20], seed=7, q_std=1.0)
    c.q.fill_(1.0)
    c.k[c.table[0, 0], 3] = torch.finfo(torch.bfloat16).min         # a key whose logit is -inf: no weight
    out, lse = _run(c)
    keep = np.arange(20) != 3
    k, v = (x[0][keep] for x in (c.own(c.k), c.own(c.v)))
    for h in range(2):
        s = c.scale * k[:, h].sum(1)
        p = np.exp(s - s.max())
        want = p @ v[:, h] / p.sum()
        assert np.abs(out[0, :, h].double().cpu().numpy() - want).max() <= 2 * UNIT["bf16"] * (np.abs(v).max() + 1)


class Sink:
    """One key of logit 16 and value 0 among n - 1 of logit 16 - below and values of about one, read by
    ``B`` sequences from the same pages: enough of them that every cache is one run of keys, or few, so
    that it is split.  All rows see the same."""

    def __init__(self, n, below, dtype, B, L=1, D=8, Hkv=8, page=256, seed=19):
        rng = np.random.default_rng(seed)
        dt = TYPES[dtype]
        pages = -(-n // page)
        k, v = torch.zeros(pages, page, Hkv, D, dtype=dt), torch.full((pages, page, Hkv, D), float("nan"), dtype=dt)
        flat_k, flat_v = k.view(-1, Hkv, D), v.view(-1, Hkv, D)
        flat_k[:, :, 0] = (16 - below) / 16
        at = n // 3
        flat_k[at, :, 0] = 1.0
        flat_v[:n] = torch.from_numpy(rng.uniform(0.5, 1.5, (n, Hkv, D))).to(dt)
        flat_v[at] = 0.0
        q = torch.zeros(B, L, Hkv, D, dtype=dt)
        q[..., 0] = 16.0
        cache = brisk.KVCache(k.cuda(), v.cuda(), torch.arange(pages, dtype=torch.int32, device="cuda").repeat(B, 1),
                              torch.full((B,), n, dtype=torch.int32, device="cuda"))
        self.out, self.lse = brisk.block_attention(q.cuda(), cache, scale=1.0)
        torch.cuda.synchronize()
        s = 16.0 * flat_k[:n, 0, 0].double().numpy()
        w = np.exp(s - s.max())
        self.want = np.tensordot(w, flat_v[:n].double().numpy(), (0, 0)) / w.sum()
        self.want_lse = s.max() + np.log(w.sum())
        assert abs(w.sum() - 1 - (n - 1) * w[0]) < 1e-9


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("L", [1, 40, 64])
def test_weak_keys_beside_a_strong_one_are_counted(dtype, L):
    """A log-sum-exp over one long run, most of it from keys whose weights are each below half a unit of the sum.

    A lane adds 16 or 32 weights, then one such sum of n / 64 tiles to the total: each addition is off by at most
    2^-25 of it.  Logits are exact."""
    n = 65537
    c = Sink(n, 17.4375, dtype, B=64, L=L)
    assert abs(c.want_lse - 16.0) > 2.0 ** -10      # what the weak keys bring
    got = c.lse.double().cpu().numpy()
    print(f"[sink] {dtype} L={L}: lse off by {np.abs(got - c.want_lse).max():.2e}", flush=True)
    assert np.abs(got - c.want_lse).max() <= (n / 64 + 32) * 2.0 ** -24 + 2.0 ** -20 * 17


@pytest.mark.parametrize("n,below,B,L", [(65537, 17.4375, 64, 1), (65537, 17.4375, 64, 40), (65537, 17.4375, 64, 64),
                                         (65537, 21.875, 64, 1), (200001, 17.4375, 64, 1), (65537, 9.0, 64, 1),
                                         (65537, 17.4375, 1, 1), (65537, 17.4375, 2, 50)])
def test_f16_probabilities_of_weak_keys(n, below, B, L):
    """Outputs that are made of keys far below the largest weight, whose own value is zero.

    Beyond the tolerance of every output (sum p |v| is the output itself here): each probability is off by at
    most 2^-37 of the largest, each of a run's n / 16 matrix products rounds its sum by 2^-24, and the output's
    own smallest step is 2^-24."""
    c = Sink(n, below, "f16", B=B, L=L)
    o = c.want
    tol = (2 * UNIT["f16"] + 2.0 ** -15 + 2 * 2.0 ** -19 * 16 + n / 16 * 2.0 ** -24) * o + n * 2.0 ** -37 * 1.5 + 2.0 ** -25
    err = np.abs(c.out.double().cpu().numpy() - o)
    print(f"[sink] n={n} below={below} B={B} L={L}: output {o.max():.2e}, off by {err.max():.2e}, may be {tol.min():.2e}", flush=True)
    assert (err <= tol).all()
    assert tol.max() < 0.1 * o.min() or below > 20  # the bound says something


@pytest.mark.parametrize("hidden", [False, True])
@pytest.mark.parametrize("kw", [
    dict(B=2, L=4, H=4, Hkv=2, D=128, prefix=70, lens=[100, 9]),
    dict(B=3, L=7, H=14, Hkv=2, D=64, prefix=None, lens=[120, 64, 7]),
    dict(B=2, L=16, H=8, Hkv=1, D=96, prefix=20, lens=[90, 30]),
    dict(B=5, L=16, H=8, Hkv=2, D=128, prefix=70, lens=[16, 40, 60, 80, 100]),
    dict(B=1, L=2, H=4, Hkv=2, D=80, prefix=40, lens=[100], dtype="f16"),
])
def test_logits_far_past_the_exponent_range(kw, hidden):
    """Finite logits whose spacing in 32 bits is many units: the largest takes all the weight.

    Every product is of two short significands, so logits are exact and the
    winner's probability is one: its value comes out bit for bit.  One head in
    two has logits of order one in the same tiles."""
    c = Case(mask="causal", seed=18, **kw)
    qs, ks = (2.0 ** 20, 2.0 ** 16) if c.dtype == "bf16" else (2.0 ** 14, 2.0 ** 14)
    for b, n in enumerate(c.lens):
        steps = c.rng.permutation(128)              # the own keys of a sequence differ
        for j in range(n):
            at = c.table[b, j // c.page], j % c.page
            c.k[at] = 0
            c.k[at][:, 0] = ks * (1 + steps[j] / 128)
        if hidden:                                  # the last position's value; only its own row may notice
            c.v[c.table[b, (n - 1) // c.page], (n - 1) % c.page] = float("inf")
    if c.prefix is not None:                        # below every own key
        c.prefix[0][:] = 0
        c.prefix[0][..., 0] = ks / 2 * (1 + torch.arange(len(c.prefix[0]))[:, None] % 128 / 128)
    c.q[..., 1:] = 0
    c.q[..., 0] = qs * (1 + torch.arange(c.L * c.H).reshape(1, c.L, c.H) % 64 / 64)
    c.q[:, :, ::2, 0] = 1 / ks
    out, lse = _run(c)
    o, z, mag, size = c.attention()
    keep = np.ones((c.B, c.L), dtype=bool)
    keep[:, -1] = not hidden
    got, log = out.double().cpu().numpy(), lse.double().cpu().numpy()
    own_k, own_v = c.own(c.k), c.own(c.v)
    G = c.H // c.Hkv
    for b in range(c.B):
        for i in np.nonzero(keep[b])[0]:
            vis = np.nonzero(ao.sees(c.lens[b], c.L, i, c.mask[b, i]))[0]
            for h in range(1, c.H, 2):
                key = own_k[b][vis, h // G, 0]
                assert (key == key.max()).sum() == 1
                win = vis[key.argmax()]
                assert np.array_equal(got[b, i, h], own_v[b][win, h // G]), (b, i, h, got[b, i, h][:4], log[b, i, h])
                assert abs(log[b, i, h] - z[b, i, h]) <= 2.0 ** -21 * abs(z[b, i, h])
    rows = np.nonzero(keep)
    small = tuple(r[rows][:, ::2] for r in (o, z, mag, size))
    _check(c, out.cpu()[rows][:, ::2], lse.cpu()[rows][:, ::2], small)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("what", ["k", "v", "both"])
@pytest.mark.parametrize("shape", [dict(B=2, L=8, H=8, Hkv=2, D=128), dict(B=9, L=31, H=7, Hkv=1, D=64),
                                   dict(B=2, L=16, H=8, Hkv=2, D=80), dict(B=2, L=31, H=4, Hkv=1, D=104),
                                   dict(B=1, L=64, H=4, Hkv=2, D=128)])
def test_hidden_slots_have_no_effect(bad, what, shape):
    """Block slots that a row does not see hold anything; rows that see them get it."""
    L = shape["L"]
    lens = [L + 3 + 30 * b for b in range(shape["B"])]
    c = Case(prefix=70, lens=lens, mask="causal", seed=8, **shape)
    clean = c.attention()
    t = L // 2                                     # rows i < t must not notice
    for b, n in enumerate(lens):
        j = n - L + t
        for x, name in ((c.k, "k"), (c.v, "v")):
            if what in (name, "both"):
                x[c.table[b, j // c.page], j % c.page] = bad
    out, lse = _run(c)
    c.L = t
    ref = tuple(r[:, :t] for r in clean)
    _check(c, out[:, :t], lse[:, :t], ref)
    if what != "k":
        assert not torch.isfinite(out[:, t:]).any()


@pytest.mark.parametrize("H", [4, 40])
def test_nan_queries_stay_in_their_rows(H):
    """A row of NaN queries is NaN, not empty; the others do not notice."""
    c = Case(2, 4, H, 2, 128, 100, [300, 40], mask="causal", seed=16)
    ref = c.attention()
    c.q[1, 2, 1, 5] = float("nan")
    out, lse = _run(c)
    assert torch.isnan(out[1, 2, 1]).all() and torch.isnan(lse[1, 2, 1])
    out[1, 2, 1], lse[1, 2, 1] = torch.from_numpy(ref[0][1, 2, 1]).to(out), float(ref[1][1, 2, 1])
    _check(c, out, lse, ref)


def test_strided_queries_and_given_buffers():
    """Queries inside a fused projection, one position of a longer block, and the caller's own buffers."""
    c = Case(3, 6, 8, 2, 128, 40, [50, 6, 33], mask="causal", seed=9)
    fused = torch.full((3, 6, 12, 136), float("nan"), dtype=torch.bfloat16, device="cuda")
    fused[:, :, 2:10, :128] = c.q.cuda()
    out = torch.empty(3, 6, 8, 128, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(3, 6, 8, device="cuda")
    ws = torch.empty(brisk.block_attention_workspace_size(3, 6, 8, 2, 128, 40, 64), dtype=torch.uint8, device="cuda")
    got = brisk.block_attention(fused[:, :, 2:10, :128], c.cache(brisk), prefix=c.gpu_prefix(),
                                block_mask=c.gpu_mask(), max_seq_len=64, out=out, lse=lse, workspace=ws)
    assert got[0] is out and got[1] is lse
    torch.cuda.synchronize()
    _check(c, out, lse)
    one = Case(3, 1, 8, 2, 128, 40, [50, 6, 33], seed=9)
    last = one.q.cuda().expand(3, 4, 8, 128).contiguous()[:, 3:]     # stride(0) of a longer block
    a = brisk.block_attention(last, one.cache(brisk), prefix=one.gpu_prefix())
    torch.cuda.synchronize()
    _check(one, *a)


@pytest.mark.parametrize("kw,q_ones,kv_ones", [
    (dict(B=1, L=1, H=1, Hkv=1, D=64, prefix=1, lens=[1], page=1, spare_pages=0), (0, 1, 2), (0, 1, 2)),
    (dict(B=3, L=1, H=4, Hkv=1, D=64, prefix=20, lens=[9, 0, 40], page=16), (1,), (2,)),
    (dict(B=2, L=3, H=1, Hkv=1, D=128, prefix=1, lens=[9, 40], page=1, mask="causal"), (2,), (1, 2)),
    (dict(B=1, L=5, H=6, Hkv=2, D=128, prefix=30, lens=[16], page=16, mask="causal", spare_pages=0), (0,), (0,)),
])
def test_strides_of_single_elements_do_not_matter(kw, q_ones, kv_ones):
    """Dimensions of one element come with whatever stride a slice or a transpose left them, keys' and values' apart."""
    c = Case(seed=33, **kw)

    def odd(t, dims, step):
        return torch.as_strided(t, t.shape, [step + i if i in dims else s for i, s in enumerate(t.stride())])

    cache = c.cache(brisk)
    assert all(cache.k_pages.shape[i] == 1 for i in kv_ones) and all(c.q.shape[i] == 1 for i in q_ones)
    cache = brisk.KVCache(odd(cache.k_pages, kv_ones, 3), odd(cache.v_pages, kv_ones, 77), cache.block_table, cache.seq_len)
    pre = c.gpu_prefix()
    ones = tuple(i for i in (0, 1) if pre[0].shape[i] == 1)
    out = brisk.block_attention(odd(c.q.cuda(), q_ones, 5), cache, prefix=(odd(pre[0], ones, 3), odd(pre[1], ones, 77)),
                                block_mask=c.gpu_mask())
    torch.cuda.synchronize()
    _check(c, *out)


def test_length_bound_and_table_are_clamped():
    """Lengths beyond the bound are cut to it, negative ones count as none, bad page ids stay inside the pool."""
    c = Case(2, 1, 4, 4, 64, None, [40, 24], seed=10, junk=0.0)
    cache = c.cache(brisk)
    cache.seq_len.copy_(torch.tensor([1000, -5], dtype=torch.int32))
    out, lse = brisk.block_attention(c.q.cuda(), cache, max_seq_len=33)
    c.lens = [33, 0]
    torch.cuda.synchronize()
    _check(c, out, lse)
    cache.block_table.fill_(-7)
    out, _ = brisk.block_attention(c.q.cuda(), cache)
    cache.block_table.fill_(1 << 30)
    brisk.block_attention(c.q.cuda(), cache)
    torch.cuda.synchronize()
    assert (out[1] == 0).all()


@pytest.mark.parametrize("prefix", [9, 0, None])
def test_zero_length_bound(prefix):
    c = Case(2, 2, 4, 4, 64, prefix, [0, 0], seed=11)
    _check(c, *_run(c, max_seq_len=0))


def test_same_bits_every_time_and_on_another_stream():
    c = Case(6, 8, 8, 2, 128, 700, [8, 900, 31, 64, 65, 2000], mask="mixed", seed=12, page=64)
    cache, q, pre, mask = c.cache(brisk), c.q.cuda(), c.gpu_prefix(), c.gpu_mask()
    a = brisk.block_attention(q, cache, prefix=pre, block_mask=mask)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ws = torch.empty(brisk.block_attention_workspace_size(6, 8, 8, 2, 128, 700, cache.max_seq_len), dtype=torch.uint8,
                     device="cuda")
    ws.fill_(0xFF)                                 # a workspace of NaN words
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        b = brisk.block_attention(q, cache, prefix=pre, block_mask=mask, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    _check(c, *b)


def test_offsets_past_32_bits():
    """Pages more than 2^31 elements (and 2^32 bytes) into the pool, and a prefix spread as wide."""
    span = 3_500_000_000 // 8 * 8                  # elements of each pool
    if torch.cuda.mem_get_info()[0] < 4 * span * 2 + (4 << 30):
        pytest.skip("needs a card with 32 GiB free")
    c = Case(1, 2, 4, 2, 128, 3, [40], mask="causal", seed=13, spare_pages=0)

    def spread(x):
        pool = torch.empty(span, dtype=torch.bfloat16, device="cuda")
        step = span // x.shape[0] // 8 * 8
        assert step * (x.shape[0] - 1) > 1 << 31
        v = pool.as_strided(x.shape, (step,) + tuple(x.stride()[1:]))
        v.copy_(x)
        return v

    cache = brisk.KVCache(spread(c.k), spread(c.v), torch.from_numpy(c.table).cuda(),
                          torch.tensor(c.lens, dtype=torch.int32).cuda())
    out, lse = brisk.block_attention(c.q.cuda(), cache, prefix=tuple(spread(x) for x in c.prefix),
                                     block_mask=c.gpu_mask())
    torch.cuda.synchronize()
    _check(c, out, lse)


def test_graph_replays():
    c = Case(4, 4, 8, 2, 128, 100, [4, 20, 300, 77], mask="causal", seed=14)
    cache, q, pre, mask = c.cache(brisk), c.q.cuda(), c.gpu_prefix(), c.gpu_mask()
    ref = brisk.block_attention(q, cache, prefix=pre, block_mask=mask)
    out, lse = torch.empty_like(ref[0]), torch.empty_like(ref[1])
    ws = torch.empty(brisk.block_attention_workspace_size(4, 4, 8, 2, 128, 100, cache.max_seq_len) + 16,
                     dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            brisk.block_attention(q, cache, prefix=pre, block_mask=mask, out=out, lse=lse, workspace=ws)
    for _ in range(4):
        out.fill_(-7)
        lse.fill_(-7)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])


@pytest.mark.parametrize("kw", [
    dict(B=3, L=7, H=6, Hkv=2, D=72, prefix=33, lens=[7, 100, 64], mask="mixed"),
    dict(B=1, L=1, H=4, Hkv=4, D=128, prefix=None, lens=[3000]),
    dict(B=20, L=8, H=8, Hkv=2, D=64, prefix=300, lens=[8 + b for b in range(20)], dtype="f16"),
])
def test_writes_stay_inside_the_buffers(kw):
    from test_gpu_canary import Guarded
    c = Case(seed=15, **kw)
    cache = c.cache(brisk)
    P = 0 if c.prefix is None else len(c.prefix[0])
    need = brisk.block_attention_workspace_size(c.B, c.L, c.H, c.Hkv, c.D, P, cache.max_seq_len)
    out = Guarded((c.B, c.L, c.H, c.D), c.q.dtype)
    lse, ws = Guarded((c.B, c.L, c.H), torch.float32), Guarded((max(need, 16),), torch.uint8)
    brisk.block_attention(c.q.cuda(), cache, prefix=c.gpu_prefix(), block_mask=c.gpu_mask(), out=out.t, lse=lse.t,
                          workspace=ws.t)
    assert out.intact() and lse.intact() and ws.intact()
    _check(c, out.t, lse.t)


def test_binding_refuses_what_does_not_fit():
    """Wrong types, shapes, strides and devices never reach the library."""
    c = Case(2, 3, 4, 2, 64, 8, [10, 20], seed=17)
    cache, q, pre = c.cache(brisk), c.q.cuda(), c.gpu_prefix()
    call = brisk.block_attention
    for bad, kw in ((q.cpu(), {}), (q[:1], {}), (q[..., :32], {}), (q[:, :, :, ::2], {}),
                    (q.transpose(0, 1).contiguous().transpose(0, 1), {}), (q, dict(prefix=(pre[0], pre[1][:, :1]))),
                    (q, dict(prefix=(pre[0], pre[1].transpose(0, 1).contiguous().transpose(0, 1)))),
                    (q, dict(block_mask=torch.zeros(2, 4, dtype=torch.int64, device="cuda"))),
                    (q, dict(out=torch.empty(2, 3, 4, 32, dtype=q.dtype, device="cuda"))),
                    (q, dict(prefix=pre, workspace=torch.empty(1, dtype=torch.uint8, device="cuda")))):
        with pytest.raises(ValueError):
            call(bad, cache, **kw)
    for bad, kw in ((q.half(), {}), (q, dict(prefix=(pre[0].half(), pre[1].half()))),
                    (q, dict(block_mask=torch.zeros(2, 3, dtype=torch.int32, device="cuda"))),
                    (q, dict(lse=torch.empty(2, 3, 4, dtype=torch.bfloat16, device="cuda")))):
        with pytest.raises(TypeError):
            call(bad, cache, **kw)
    with pytest.raises(brisk.BriskError) as e:
        call(q, cache, scale=-1.0)
    assert e.value.status == -2
    with pytest.raises(brisk.BriskError):
        call(q, cache, max_seq_len=cache.max_seq_len + 1)
    k = cache.k_pages
    with pytest.raises(ValueError):
        brisk.KVCache(k, k[:, :8], cache.block_table, cache.seq_len)
    with pytest.raises(ValueError):
        brisk.KVCache(k, k, cache.block_table, cache.seq_len[:1])
