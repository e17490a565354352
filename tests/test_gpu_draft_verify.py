"""GPU checks of brisk_draft_verify against the float64 oracle: accepted
lengths and drawn tokens are equal wherever 32-bit rounding cannot decide
(the oracle says where it can), and the committed token follows the target."""
import numpy as np
import pytest
import torch
from scipy import stats

import oracle.attention_oracle as ao

pytestmark = pytest.mark.gpu

brisk = pytest.importorskip("paper_2609_33390_amd")


def _laws(B, L, V, rng, std=2.0, noise=0.7):
    z = std * rng.standard_normal((B, L + 1, V))
    d = z[:, :L] + noise * rng.standard_normal((B, L, V))
    soft = lambda x: (np.exp(x - x.max(-1, keepdims=True)) / np.exp(x - x.max(-1, keepdims=True)).sum(-1, keepdims=True))  # noqa: E731
    target, draft = soft(z).astype(np.float32), (soft(d) if L else d).astype(np.float32)
    tok = np.array([[rng.choice(V, p=draft[b, i].astype(np.float64) / draft[b, i].astype(np.float64).sum())
                     for i in range(L)] for b in range(B)], dtype=np.int32).reshape(B, L)
    return target, draft, tok, rng.random((B, L)).astype(np.float32), rng.exponential(size=(B, V)).astype(np.float32)


def _gpu(target, draft, tok, u, noise, n=None, **kw):
    t = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    a, x = brisk.draft_verify(t(target), t(draft), t(tok), t(u), t(noise), draft_len=None if n is None else t(n), **kw)
    torch.cuda.synchronize()
    return a.cpu().numpy(), x.cpu().numpy()


def _compare(target, draft, tok, u, noise, n, got):
    sure = 0
    for b in range(len(noise)):
        a, x, close = ao.draft_verify(target[b], draft[b], tok[b], tok.shape[1] if n is None else int(n[b]), u[b], noise[b])
        if not close:
            sure += 1
            assert (got[0][b], got[1][b]) == (a, x), b
    assert sure >= 0.9 * len(noise)


@pytest.mark.parametrize("B,L,V,ragged", [
    (1, 1, 1, False), (1, 8, 1003, False), (3, 1, 2, False), (5, 0, 517, False), (70, 4, 333, True), (2, 64, 5000, True),
    (3, 70, 129, False), (1, 3, 126464, False), (17, 5, 20001, True), (600, 3, 640, True), (2, 16, 65537, False),
])
def test_draft_verify_matches_oracle(B, L, V, ragged):
    print(f"[draft] B={B} L={L} V={V}", flush=True)
    rng = np.random.default_rng(B * 1000 + L)
    target, draft, tok, u, noise = _laws(B, L, V, rng)
    n = rng.integers(-1, L + 2, B).astype(np.int32) if ragged else None
    got = _gpu(target, draft, tok, u, noise, n)
    _compare(target, draft, tok, u, noise, None if n is None else np.clip(n, 0, L), got)


def test_same_laws_accept_everything():
    rng = np.random.default_rng(1)
    target, _, tok, u, noise = _laws(6, 5, 300, rng)
    draft = target[:, :5].copy()
    got = _gpu(target, draft, tok, u, noise)
    assert (got[0] == 5).all()
    _compare(target, draft, tok, u, noise, None, got)


def test_one_hot_target_is_greedy_verification():
    rng = np.random.default_rng(2)
    B, L, V = 40, 6, 257
    _, draft, tok, u, noise = _laws(B, L, V, rng)
    best = rng.integers(0, V, (B, L + 1))
    best[:, :L] = np.where(rng.random((B, L)) < 0.7, tok, best[:, :L])
    target = np.zeros((B, L + 1, V), dtype=np.float32)
    np.put_along_axis(target, best[..., None], 1.0, -1)
    got = _gpu(target, draft, tok, u, noise)
    acc, cor = brisk.verify_accept(torch.from_numpy(tok).cuda(), torch.from_numpy(best[:, :L].astype(np.int32)).cuda())
    assert np.array_equal(got[0], acc.cpu().numpy())
    want = np.where(got[0] < L, cor.cpu().numpy(), best[:, L])
    assert np.array_equal(got[1], want)


def test_empty_rows_ties_and_strange_weights():
    """No positive weight: -1.  Ties: the lower id.  NaN and negative weights are never drawn.  A rejection
    whose difference is positive nowhere draws from the target itself."""
    V = 700
    noise = np.ones((6, V), dtype=np.float32)
    target = np.zeros((6, 2, V), dtype=np.float32)
    draft = np.full((6, 1, V), 0.5, dtype=np.float32)
    tok = np.zeros((6, 1), dtype=np.int32)
    u = np.full((6, 1), 0.9, dtype=np.float32)
    target[1, 0, [650, 300, 301]] = 0.25           # below the draft everywhere: from the target, lowest of the tie
    target[2, 0, 1:] = np.nan
    target[2, 0, 5] = 0.75
    target[3, 0, 699] = 1.0
    target[3, 0, 2] = -3.0
    target[4, 0, 0] = 0.46                         # 0.9 * 0.5 < 0.46: accepted, then an empty row
    target[5, 0, 0], target[5, 1, 698], noise[5, 698] = 0.46, 1e-30, 1e30     # the ratio underflows to zero
    got = _gpu(target, draft, tok, u, noise)
    assert got[0].tolist() == [0, 0, 0, 0, 1, 1]
    assert got[1].tolist() == [-1, 300, 5, 699, -1, -1]


def test_strided_rows_and_bad_tokens():
    """Rows padded past V and unaligned, tokens outside the vocabulary, negative and oversized draft lengths."""
    rng = np.random.default_rng(3)
    B, L, V = 9, 4, 1001
    target, draft, tok, u, noise = _laws(B, L, V, rng)
    pad = lambda x, w: torch.full(x.shape[:-1] + (w,), float("nan"), device="cuda")  # noqa: E731
    T, D, N = pad(target, V + 7), pad(draft, V + 1), pad(noise, V + 2)
    for wide, x in ((T, target), (D, draft), (N, noise)):
        wide[..., 1:1 + V] = torch.from_numpy(x).cuda()
    n = np.array([-3, 9, 0, 1, 2, 3, 4, 4, 4], dtype=np.int32)
    t = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    a, x = brisk.draft_verify(T[..., 1:1 + V], D[..., 1:1 + V], t(tok), t(u), N[..., 1:1 + V], draft_len=t(n))
    torch.cuda.synchronize()
    _compare(target, draft, tok, u, noise, np.clip(n, 0, L), (a.cpu().numpy(), x.cpu().numpy()))
    tok[:, 0] = [-5, 1 << 30] * 4 + [V]
    a, x = _gpu(target, draft, tok, u, noise)
    assert ((a >= 0) & (a <= L) & (x >= 0) & (x < V)).all()


def test_committed_token_follows_the_target():
    """First committed token of each block against the target's first row, by chi-squared."""
    rng = np.random.default_rng(4)
    B, V = 60000, 13
    target1, draft1, _, _, _ = _laws(1, 1, V, rng, std=1.0, noise=1.0)
    p, q = target1[0, 0].astype(np.float64), draft1[0, 0].astype(np.float64)
    tok = rng.choice(V, size=(B, 1), p=q / q.sum()).astype(np.int32)
    u, noise = rng.random((B, 1)).astype(np.float32), rng.exponential(size=(B, V)).astype(np.float32)
    a, x = _gpu(np.repeat(target1, B, 0), np.repeat(draft1, B, 0), tok, u, noise)
    first = np.where(a > 0, tok[:, 0], x)
    count = np.bincount(first, minlength=V)
    assert stats.chisquare(count, p / p.sum() * B).pvalue > 1e-4


def test_graph_and_guard_bands():
    from test_gpu_canary import Guarded
    import ctypes
    rng = np.random.default_rng(5)
    B, L, V = 5, 4, 30011
    laws = _laws(B, L, V, rng)
    t = [torch.from_numpy(x).cuda() for x in laws]
    nbytes = ctypes.c_size_t()
    assert brisk.lib().brisk_draft_verify_workspace_size(B, V, ctypes.byref(nbytes)) == 0
    acc, tok, ws = Guarded((B,), torch.int32), Guarded((B,), torch.int32), Guarded((max(16, nbytes.value),), torch.uint8)
    call = lambda: brisk.draft_verify(*t, accept_len=acc.t, token=tok.t, workspace=ws.t)  # noqa: E731
    call()
    assert acc.intact() and tok.intact() and ws.intact()
    ref = acc.t.clone(), tok.t.clone()
    _compare(*laws, None, tuple(x.cpu().numpy() for x in ref))
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            call()
    for _ in range(4):
        acc.t.fill_(-9)
        tok.t.fill_(-9)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(acc.t, ref[0]) and torch.equal(tok.t, ref[1])


def test_binding_refuses_what_does_not_fit():
    rng = np.random.default_rng(6)
    t, d, x, u, e = (torch.from_numpy(v).cuda() for v in _laws(3, 4, 50, rng))
    call = brisk.draft_verify
    for args in ((t[:, :4], d, x, u, e), (t, d[:, :3], x, u, e), (t, d, x, u[:2], e), (t, d, x, u, e[:, :49]),
                 (t[..., ::2], d, x, u, e), (t.cpu(), d, x, u, e), (t[0], d, x, u, e)):
        with pytest.raises(ValueError):
            call(*args)
    for args in ((t.double(), d, x, u, e), (t, d.half(), x, u, e), (t, d, x.long(), u, e)):
        with pytest.raises(TypeError):
            call(*args)
    with pytest.raises(ValueError):
        call(t, d, x, u, e, draft_len=torch.zeros(2, dtype=torch.int32, device="cuda"))
