"""Calls that bring no workspace, on several streams and under capture (GPU)."""
import pytest
import torch

from kv_cases import Case

pytestmark = pytest.mark.gpu

brisk = pytest.importorskip("paper_2609_33390_amd")


def _attend_calls():
    """Attention calls of different shapes, all split into runs that meet in scratch."""
    calls = []
    for kw in (dict(B=6, L=8, H=8, Hkv=2, D=128, prefix=700, lens=[8, 900, 31, 64, 65, 2000], mask="mixed", page=64),
               dict(B=1, L=1, H=8, Hkv=8, D=128, prefix=None, lens=[9001], page=64),
               dict(B=2, L=8, H=8, Hkv=2, D=64, prefix=5000, lens=[6000, 37], mask="causal", page=256, dtype="f16")):
        c = Case(seed=30, junk=0.0, **kw)
        args = (c.q.cuda(), c.cache(brisk))
        more = dict(prefix=c.gpu_prefix(), block_mask=c.gpu_mask())
        calls.append(lambda args=args, more=more, **kw: brisk.block_attention(*args, **more, **kw))
    return calls


def _evict_calls():
    """Evictions of different shapes, one of them with the scratch of long caches."""
    calls = []
    for lens, budget, Hkv in (([900, 300], 100, 4), ([40000, 33], 20000, 2), ([2500], 1000, 8)):
        c = Case(len(lens), 1, Hkv, Hkv, 16, None, lens, junk=0.0, seed=31)
        cap = max(lens)
        score = torch.from_numpy(c.rng.random((c.B, Hkv, cap))).float().cuda()
        pos = torch.arange(cap, dtype=torch.int32, device="cuda").expand(c.B, Hkv, cap).contiguous()
        at = torch.tensor(lens, dtype=torch.int32, device="cuda")
        cache = c.cache(brisk)                      # the sources stay, so each call moves the same rows
        calls.append(lambda a=(cache, score, pos, at, budget, 10), **kw: (*brisk.cache_evict(*a, **kw), a[0].k_pages, a[0].v_pages))
    return calls


@pytest.mark.parametrize("calls", [_attend_calls, _evict_calls])
@pytest.mark.parametrize("how", ["current", "argument", "handle"])
def test_interleaved_streams_without_workspaces(calls, how):
    calls = calls()
    want = [[x.clone() for x in f()] for f in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    got = [[] for _ in calls]
    for turn in range(6):
        for i, (f, s) in enumerate(zip(calls, streams)):
            if how == "current":
                with torch.cuda.stream(s):
                    got[i].append(f())
            else:
                got[i].append(f(stream=s if how == "argument" else s.cuda_stream))
    torch.cuda.synchronize()
    for i, w in enumerate(want):
        for out in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(out, w))


def test_graph_without_a_workspace_beside_larger_calls():
    """A captured call keeps its scratch: larger eager calls of the same kind in between change nothing."""
    small, large = _attend_calls()[1], _attend_calls()[2]
    want = [x.clone() for x in small()]
    out, lse = (torch.empty_like(x) for x in want)
    torch.cuda.synchronize()
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            small(out=out, lse=lse)
    for _ in range(4):
        out.fill_(-7)
        lse.fill_(-7)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            large()
            torch.full((1 << 20,), float("nan"), device="cuda")
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
