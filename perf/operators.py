"""Timing cases of the operators around a decoding step: the attention of a
block over a shared prefix and a paged cache, the two halves of that cache's
eviction, and the verification of drafted tokens against given probabilities.

A case is a dict of plain values.  ``op`` names the operator:

  attend   B sequences of L positions, H query heads on Hkv key/value heads of
           D elements, ``prefix`` shared keys, own lengths spread from ``lo``
           to ``hi`` keys (the last L of them the block itself, seen through
           ``mask``), pages of ``page`` tokens in ``layout`` order
  score    the attention weight every cached key received, added to its score
  evict    at most ``budget`` keys a head stay, the ``recent`` latest for certain
  verify   B drafts of up to L tokens over V words

Where ``own`` is false, ``run`` computes each operator from elementary torch
operations in 32 bits; where it is true, it calls the framework.  ``exact``
gives the same outputs from the definitions in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
OPS = ("attend", "score", "evict", "verify")
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def _attend(name, B, L, H, Hkv, D, prefix, lo, hi, mask="full", page=64, layout="nhd", dtype="bf16", op="attend"):
    return dict(name=name, op=op, B=B, L=L, H=H, Hkv=Hkv, D=D, prefix=prefix, lo=lo, hi=hi, mask=mask, page=page,
                layout=layout, dtype=dtype)


def listed():
    return [
        # one request, one token at a time: the smallest call, where latency counts
        _attend("attend-b1-l1-n1500", 1, 1, 32, 8, 128, 0, 1500, 1500, page=16),
        # one request's block deep in a long document: one long cache, few rows
        _attend("attend-b1-l32-n65k", 1, 32, 32, 8, 128, 0, 65568, 65568),
        # single tokens of many requests that share a long system prompt
        _attend("attend-b256-l1-p4k", 256, 1, 28, 4, 128, 4096, 1, 512, page=16),
        # the largest: blocks of many requests over a shared document and their own ragged contexts,
        # verified positions (causal) and masked ones (bidirectional) in one block
        _attend("attend-b64-l16-p16k", 64, 16, 32, 8, 128, 16384, 16, 2048, mask="mixed"),
        # blocks of a model that has a key head for each query head, no shared prefix
        _attend("attend-b32-l32-mha", 32, 32, 32, 32, 128, 0, 40, 1100, mask="causal"),
        # odd sizes throughout: another type, a narrow head, head-major pages, a ragged prefix
        _attend("attend-b13-l21-d80", 13, 21, 30, 6, 80, 1003, 5, 777, mask="mixed", page=32, layout="hnd", dtype="f16"),
        # scores of a serving batch's caches after a block
        _attend("score-b64-l16", 64, 16, 32, 8, 128, 0, 500, 4000, mask="mixed", op="score"),
        # scores of one long cache after one token, a narrow head
        _attend("score-b1-l1-n33k", 1, 1, 16, 4, 64, 0, 33001, 33001, page=16, dtype="f16", op="score"),
        # a serving batch whose caches have outgrown their budget, some not yet
        dict(name="evict-b64-n4k", op="evict", B=64, Hkv=8, D=128, lo=1800, hi=4100, budget=2048, recent=128, page=64,
             layout="nhd", dtype="bf16"),
        # one long cache cut to a quarter
        dict(name="evict-b1-n120k", op="evict", B=1, Hkv=4, D=128, lo=120001, hi=120001, budget=30000, recent=1000,
             page=16, layout="hnd", dtype="f16"),
        # one request's draft: latency
        dict(name="verify-b1-l8", op="verify", B=1, L=8, V=126464, ragged=False),
        # a large batch of drafts of different lengths, the wide vocabulary
        dict(name="verify-b128-l7", op="verify", B=128, L=7, V=152064, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_one(rng):
    op = rng.choice(("attend", "attend", "attend", "score", "evict", "verify"))
    if op == "verify":
        return dict(op=op, B=_log_int(rng, 1, 128), L=rng.randint(1, 16), V=_log_int(rng, 2000, 152064),
                    ragged=rng.random() < 0.5)
    c = dict(op=op, B=_log_int(rng, 1, 256), D=rng.choice((64, 80, 96, 128, 128)), page=rng.choice((16, 32, 64, 128)),
             layout=rng.choice(("nhd", "hnd")), dtype=rng.choice(("bf16", "bf16", "f16")))
    if op == "evict":
        c["Hkv"] = rng.choice((1, 2, 4, 8, 32))
        c["hi"] = _log_int(rng, 64, 120000)
        c["lo"] = rng.randint(c["hi"] // 2, c["hi"])
        c["budget"] = rng.randint(c["hi"] // 8, c["hi"])
        c["recent"] = rng.randint(0, c["budget"] // 4)
        return c
    Hkv, G = rng.choice(((8, 4), (4, 7), (32, 1), (2, 8), (6, 5), (1, 16)))
    c.update(L=rng.choice((1, 1, 7, 8, 16, 32, rng.randint(2, 64))), H=Hkv * G, Hkv=Hkv,
             prefix=0 if op == "score" or rng.random() < 0.4 else _log_int(rng, 1, 16384),
             mask=rng.choice(("full", "causal", "mixed")))
    c["hi"] = _log_int(rng, 4, 65568)
    c["lo"] = rng.randint(0, c["hi"])
    return c


def draw(rng):
    top = [work(c) for c in listed()]
    while True:
        c = _draw_one(rng)
        w = work(c)
        pairs = c["B"] * c["L"] * c["H"] * (c["prefix"] + c["hi"]) if "prefix" in c else 0
        if (w["bytes"] <= max(t["bytes"] for t in top) and w["flops"] <= max(t["flops"] for t in top)
                and pairs <= 600_000_000 and c["B"] * c.get("Hkv", 1) * c.get("hi", 1) <= 3_000_000
                and 3072 not in c.values()):
            return c


def _lengths(c):
    """Own lengths spread evenly from lo to hi."""
    if c["B"] == 1:
        return [c["hi"]]
    return [c["lo"] + (c["hi"] - c["lo"]) * b // (c["B"] - 1) for b in range(c["B"])]


def work(case):
    c, B = case, case["B"]
    if c["op"] == "verify":
        # two probabilities a position, then one row of target, draft and noise a block
        return {"bytes": B * (c["L"] * 16 + 12 * c["V"] + 8), "flops": 4 * B * c["V"]}
    n = sum(_lengths(c))
    if c["op"] == "evict":
        moved = sum(max(0, x - c["budget"]) * c["budget"] / max(1, x) for x in _lengths(c)) * c["Hkv"]
        return {"bytes": 8 * c["Hkv"] * (n + B * min(c["budget"], c["hi"])) + 8 * c["D"] * moved, "flops": c["Hkv"] * n}
    rows = B * c["L"] * c["H"]
    if c["op"] == "score":
        return {"bytes": 2 * c["Hkv"] * c["D"] * n + rows * (2 * c["D"] + 4) + 8 * c["Hkv"] * n + 8 * B,
                "flops": 2 * c["L"] * c["H"] * c["D"] * n}
    return {"bytes": 4 * c["Hkv"] * c["D"] * (c["prefix"] + n) + rows * (4 * c["D"] + 4) + 8 * B,
            "flops": 4 * c["L"] * c["H"] * c["D"] * (B * c["prefix"] + n)}


# ------------------------------------------------------------------- inputs
def _pages(c, lens, g):
    """Paged keys and values of the sequences' own tokens, their pages in no order."""
    ps, Hkv, D, dt = c["page"], c["Hkv"], c["D"], TYPES[c["dtype"]]
    need = [-(-n // ps) for n in lens]
    n_pages, most = sum(need) + 3, max(1, max(need))
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    start = torch.tensor([sum(need[:b]) for b in range(len(need))], device=DEV)
    col = torch.arange(most, device=DEV)
    table = order[torch.clamp(start[:, None] + col[None], max=n_pages - 1)].contiguous()
    shape = (n_pages, ps, Hkv, D) if c["layout"] == "nhd" else (n_pages, Hkv, ps, D)
    k, v = (torch.randn(shape, generator=g, device=DEV).to(dt) for _ in range(2))
    if c["layout"] == "hnd":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    return dict(k=k, v=v, table=table, seq_len=torch.tensor(lens, dtype=torch.int32, device=DEV))


def _block_mask(c, lens):
    """Bit t of row i: position i of the block sees its position t."""
    L = c["L"]
    if c["mask"] == "full":
        return None
    half = L if c["mask"] == "causal" else (L + 1) // 2
    rows = [(1 << (i + 1)) - 1 if i < half else (1 << L) - 1 for i in range(L)]
    rows = [r - (1 << 64) if r >= 1 << 63 else r for r in rows]
    return torch.tensor(rows, dtype=torch.int64, device=DEV).repeat(len(lens), 1)


def prepare(case, seed):
    c, B = case, case["B"]
    g = torch.Generator(device=DEV)
    g.manual_seed(1_000_003 * (seed + 1) + OPS.index(c["op"]))
    if c["op"] == "verify":
        return _prepare_verify(c, g)
    order = torch.randperm(B, generator=g, device=DEV).tolist()
    lens = [_lengths(c)[b] for b in order]
    s = dict(case=c, **_pages(c, lens, g))
    if own:
        import paper_2609_33390_amd as brisk
        s["cache"] = brisk.KVCache(s["k"], s["v"], s["table"], s["seq_len"])
    if c["op"] == "evict":
        return _prepare_evict(c, s, lens, g)
    L, H, Hkv, D, dt = c["L"], c["H"], c["Hkv"], c["D"], TYPES[c["dtype"]]
    # the queries are the first columns of the layer's fused projection; scores of about +-2 after the scale
    s["q"] = (2.0 * torch.randn(B, L, H + 2 * Hkv, D, generator=g, device=DEV)).to(dt)[:, :, :H]
    s["mask"] = _block_mask(c, lens)
    s["scale"] = D ** -0.5
    if c["op"] == "attend":
        s["prefix"] = None
        if c["prefix"]:
            shape = (c["prefix"], Hkv, D) if c["layout"] == "nhd" else (Hkv, c["prefix"], D)
            kv = [torch.randn(shape, generator=g, device=DEV).to(dt) for _ in range(2)]
            s["prefix"] = tuple(t if c["layout"] == "nhd" else t.transpose(0, 1) for t in kv)
        return s
    # the attention before it left the log-sum-exp of every row, part of it over keys that are not in this cache
    most = max(1, max(lens))
    z, vis = _own_logits(s, most)
    lse = torch.logsumexp(z.masked_fill(~vis, -math.inf), dim=-1).transpose(1, 2)
    s["lse"] = (lse + 0.3 * torch.rand(lse.shape, generator=g, device=DEV)).contiguous()
    s["score"] = torch.rand(B, Hkv, s["table"].shape[1] * c["page"], generator=g, device=DEV) * 0.1
    s["decay"] = 0.96875
    return s


def _prepare_evict(c, s, lens, g):
    B, Hkv = c["B"], c["Hkv"]
    cap = s["table"].shape[1] * c["page"]
    # accumulated weights: a few keys hold most of it, some never got any
    score = torch.randn(B, Hkv, cap, generator=g, device=DEV).mul_(1.5).exp_()
    score *= (torch.rand(B, Hkv, cap, generator=g, device=DEV) > 0.05)
    # earlier evictions left gaps, and the older half of the slots in no order
    n = torch.tensor(lens, device=DEV)
    slot = torch.arange(cap, device=DEV)
    gone = 500
    old = slot[None] < (n // 2)[:, None]
    shuffled = torch.rand(B, Hkv, cap, generator=g, device=DEV).masked_fill(~old[:, None], 2.0).argsort(-1)
    pos = torch.where(old[:, None], shuffled, (slot + gone)[None, None])
    s.update(score=score, pos=pos.to(torch.int32).contiguous(), next_pos=(n + gone).to(torch.int32))
    return s


def _prepare_verify(c, g):
    B, L, V = c["B"], c["L"], c["V"]
    target = torch.randn(B, L + 1, V, generator=g, device=DEV).mul_(2.5)
    draft = target[:, :L] + 0.6 * torch.randn(B, L, V, generator=g, device=DEV)
    target, draft = torch.softmax(target, -1), torch.softmax(draft, -1)
    # the draft's own tokens, drawn from its law
    e = torch.empty(B, V, device=DEV)
    tok = torch.stack([(draft[:, i] / e.exponential_(generator=g)).argmax(-1) for i in range(L)], 1).to(torch.int32)
    n = torch.randint(0, L + 1, (B,), generator=g, device=DEV, dtype=torch.int32) if c["ragged"] else None
    return dict(case=c, target=target, draft=draft, tok=tok, draft_len=n, u=torch.rand(B, L, generator=g, device=DEV),
                noise=torch.empty(B, V, device=DEV).exponential_(generator=g))


# -------------------------------------------------------------------- passes
def run(state):
    return (_framework if own else _plain)(state)


def _framework(s):
    import paper_2609_33390_amd as brisk
    op = s["case"]["op"]
    if op == "attend":
        out, lse = brisk.block_attention(s["q"], s["cache"], prefix=s["prefix"], block_mask=s["mask"], scale=s["scale"])
        return dict(out=out, lse=lse)
    if op == "score":
        return dict(score=brisk.cache_score(s["q"], s["lse"], s["cache"], s["score"], block_mask=s["mask"],
                                            scale=s["scale"], decay=s["decay"]))
    if op == "evict":
        c = s["case"]
        score, pos, n = brisk.cache_evict(s["cache"], s["score"], s["pos"], s["next_pos"], c["budget"], c["recent"])
        return dict(score=score, pos=pos, n=n, k=s["k"], v=s["v"])
    accept, token = brisk.draft_verify(s["target"], s["draft"], s["tok"], s["u"], s["noise"], draft_len=s["draft_len"])
    return dict(accept=accept, token=token)


def _plain(s):
    return {"attend": _plain_attend, "score": _plain_score, "evict": _plain_evict, "verify": _plain_verify}[s["case"]["op"]](s)


def _own_rows(s, x, most):
    """[B, Hkv, most, D] of a page array, in 32 bits."""
    j = torch.arange(most, device=DEV)
    page = s["table"][:, j // s["case"]["page"]].long()
    return x[page, (j % s["case"]["page"])[None]].float().transpose(1, 2)


def _visible(s, most):
    """[B, L, most]: the keys of the cache that a position sees."""
    c, n = s["case"], s["seq_len"].long()
    j = torch.arange(most, device=DEV)
    t = j[None] - (n - c["L"])[:, None]
    if s["mask"] is None:
        vis = torch.ones(c["B"], c["L"], most, dtype=torch.bool, device=DEV)
    else:
        vis = (t < 0)[:, None] | (((s["mask"][:, :, None] >> t.clamp(0, 63)[:, None]) & 1) == 1)
    return vis & (j[None] < n[:, None])[:, None]


def _grouped_q(s):
    """[B, Hkv, G * L, D] in 32 bits, scaled."""
    c = s["case"]
    q = s["q"].float() * s["scale"]
    return q.transpose(1, 2).reshape(c["B"], c["Hkv"], -1, c["D"])


def _own_logits(s, most):
    """[B, H, L, most] logits of the own keys, [B, 1, L, most] their visibility."""
    c = s["case"]
    z = torch.matmul(_grouped_q(s), _own_rows(s, s["k"], most).transpose(-1, -2))
    return z.reshape(c["B"], c["H"], c["L"], most), _visible(s, most)[:, None]


def _plain_attend(s):
    c = s["case"]
    B, L, H, Hkv, D = c["B"], c["L"], c["H"], c["Hkv"], c["D"]
    most = max(1, c["hi"])
    z, vis = _own_logits(s, most)                                    # [B, H, L, most]
    z = z.masked_fill(~vis, -math.inf)
    m = z.amax(-1, keepdim=True)
    if s["prefix"] is not None:
        kp, vp = (t.float().transpose(0, 1) for t in s["prefix"])    # [Hkv, P, D]
        to_heads = lambda t: t.reshape(Hkv, B, H // Hkv, L, -1).transpose(0, 1).reshape(B, H, L, -1)  # noqa: E731
        zp = torch.matmul(_grouped_q(s).transpose(0, 1).reshape(Hkv, -1, D), kp.transpose(-1, -2))
        m = torch.maximum(m, to_heads(zp.amax(-1)))
    m = m.masked_fill(m == -math.inf, 0.0)
    p = torch.exp(z - m)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(B, Hkv, -1, most), _own_rows(s, s["v"], most)).reshape(B, H, L, D)
    if s["prefix"] is not None:
        pp = torch.exp(zp - m.reshape(B, Hkv, -1, 1).transpose(0, 1).reshape(Hkv, -1, 1))
        total = total + to_heads(pp.sum(-1))
        o = o + to_heads(torch.matmul(pp, vp))
    out = torch.where(total > 0, o / total, torch.zeros_like(o))
    lse = torch.where(total > 0, m + torch.log(total), torch.full_like(total, -math.inf))
    return dict(out=out.transpose(1, 2).to(TYPES[c["dtype"]]), lse=lse[..., 0].transpose(1, 2))


def _plain_score(s):
    c = s["case"]
    B, L, H, Hkv = c["B"], c["L"], c["H"], c["Hkv"]
    most = max(1, c["hi"])
    z, vis = _own_logits(s, most)                                    # [B, H, L, most]
    lse = s["lse"].transpose(1, 2)[..., None]                        # [B, H, L, 1]
    p = torch.where(vis & (lse > -math.inf), torch.exp(z - lse), torch.zeros_like(z))
    new = p.reshape(B, Hkv, H // Hkv * L, most).sum(2)
    out = torch.zeros_like(s["score"])
    held = torch.arange(most, device=DEV)[None, None] < s["seq_len"][:, None, None]
    out[:, :, :most] = torch.where(held, s["decay"] * s["score"][:, :, :most] + new, torch.zeros_like(new))
    return dict(score=out)


def _plain_evict(s):
    c = s["case"]
    n, cap, ps = s["seq_len"].long()[:, None, None], s["score"].shape[2], c["page"]
    budget = min(c["budget"], cap)
    slot = torch.arange(cap, device=DEV)[None, None]
    late = s["pos"] >= (s["next_pos"] - c["recent"])[:, None, None]
    key = torch.where(late, torch.full_like(s["score"], math.inf), s["score"])
    key = torch.where(slot < n, key, torch.full_like(key, -math.inf))
    best = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :budget]
    keep = torch.zeros_like(key, dtype=torch.bool).scatter_(-1, best, True) & (slot < n)
    full = n > budget
    src, dst = (keep & (slot >= budget) & full).nonzero(), (~keep & (slot < budget) & full).nonzero()
    b, h = src[:, 0], src[:, 1]
    page = lambda j: (s["table"][b, j // ps].long(), j % ps, h)      # noqa: E731
    for x in (s["k"], s["v"]):
        x[page(dst[:, 2])] = x[page(src[:, 2])]
    new_n = torch.minimum(n, torch.full_like(n, budget))
    score, pos = s["score"].clone(), s["pos"].clone()
    score[b, h, dst[:, 2]] = s["score"][b, h, src[:, 2]]
    pos[b, h, dst[:, 2]] = s["pos"][b, h, src[:, 2]]
    score = score.masked_fill(slot >= new_n, 0.0)
    pos = pos.masked_fill(slot >= new_n, -1)
    return dict(score=score, pos=pos, n=new_n[:, 0, 0].to(torch.int32), k=s["k"], v=s["v"])


def _plain_verify(s):
    c = s["case"]
    B, L = c["B"], c["L"]
    tok, b = s["tok"].long()[..., None], torch.arange(B, device=DEV)
    p, q = (s[x][:, :L].gather(-1, tok)[..., 0] for x in ("target", "draft"))
    n = torch.full((B,), L, device=DEV) if s["draft_len"] is None else s["draft_len"].long()
    ok = (s["u"] * q < p) & (torch.arange(L, device=DEV)[None] < n[:, None])
    a = torch.cumprod(ok.long(), 1).sum(1)
    pr = s["target"][b, a]
    w = torch.where((a < n)[:, None], pr - s["draft"][b, a.clamp(max=L - 1)], pr)
    w = torch.where((w > 0).any(-1, keepdim=True), w, pr)
    ratio = torch.where(w > 0, w / s["noise"], torch.zeros_like(w))
    best = ratio.amax(-1, keepdim=True)
    first = (ratio == best).long().argmax(-1)
    token = torch.where(best[:, 0] > 0, first, torch.full_like(first, -1))
    return dict(accept=a.to(torch.int32), token=token.to(torch.int32))


# --------------------------------------------------------------- definitions
def exact(case, seed):
    """The outputs of one pass in 64 bits, one sequence or block at a time."""
    s = prepare(case, seed)
    return {"attend": _exact_attend, "score": _exact_score, "evict": _exact_evict, "verify": _exact_verify}[case["op"]](s)


def _keys_of(s, x, b, n):
    """[Hkv, n, D] of sequence b in 64 bits."""
    ps = s["case"]["page"]
    flat = x[s["table"][b, :max(1, -(-n // ps))].long()]
    return flat.reshape(-1, x.shape[2], x.shape[3])[:n].double().permute(1, 0, 2).contiguous()


def _sees(s, b, n):
    """[L, n] of sequence b."""
    L = s["case"]["L"]
    sees = torch.ones(L, n, dtype=torch.bool, device=DEV)
    if s["mask"] is not None:
        rows = s["mask"][b].tolist()
        for t in range(L):
            j = n - L + t
            if j >= 0:
                sees[:, j] = torch.tensor([bool((r >> t) & 1) for r in rows], device=DEV)
    return sees


def _logits_of(s, b, k):
    """[H, L, keys]: 64-bit scaled products of sequence b's rows with the keys."""
    G = s["case"]["H"] // s["case"]["Hkv"]
    q = s["q"][b].double().permute(1, 0, 2).contiguous() * s["scale"]
    return torch.stack([q[h] @ k[h // G].T for h in range(s["case"]["H"])])


def _exact_attend(s):
    c = s["case"]
    G = c["H"] // c["Hkv"]
    pre = None if s["prefix"] is None else [t.double().permute(1, 0, 2).contiguous() for t in s["prefix"]]
    outs, lses = [], []
    for b, n in enumerate(s["seq_len"].tolist()):
        k, v = _keys_of(s, s["k"], b, n), _keys_of(s, s["v"], b, n)
        sees = _sees(s, b, n)
        if pre is not None:
            k, v = torch.cat([pre[0], k], 1), torch.cat([pre[1], v], 1)
            sees = torch.cat([torch.ones(c["L"], c["prefix"], dtype=torch.bool, device=DEV), sees], 1)
        z = _logits_of(s, b, k).masked_fill(~sees[None], -math.inf)
        lse = torch.logsumexp(z, -1) if z.shape[-1] else torch.full(z.shape[:2], -math.inf, device=DEV, dtype=torch.float64)
        w = torch.where(lse[..., None] > -math.inf, torch.exp(z - lse[..., None]), torch.zeros_like(z))
        outs.append(torch.stack([w[h] @ v[h // G] for h in range(c["H"])], 1))
        lses.append(lse.T)
    return dict(out=torch.stack(outs), lse=torch.stack(lses))


def _exact_score(s):
    c = s["case"]
    out = torch.zeros(s["score"].shape, dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["seq_len"].tolist()):
        if n == 0:
            continue
        z = _logits_of(s, b, _keys_of(s, s["k"], b, n))
        lse = s["lse"][b].double().T[..., None]
        w = torch.where(_sees(s, b, n)[None] & (lse > -math.inf), torch.exp(z - lse), torch.zeros_like(z))
        out[b, :, :n] = s["decay"] * s["score"][b, :, :n].double() + w.reshape(c["Hkv"], -1, n).sum(1)
    return dict(score=out)


def _exact_evict(s):
    c, ps = s["case"], s["case"]["page"]
    score, pos, new_n = s["score"].double(), s["pos"].clone(), []
    k, v = s["k"], s["v"]
    for b, n in enumerate(s["seq_len"].tolist()):
        m = min(n, c["budget"])
        new_n.append(m)
        for h in range(c["Hkv"] if n > m else 0):
            late = s["pos"][b, h, :n] >= s["next_pos"][b] - c["recent"]
            rank = torch.argsort(s["score"][b, h, :n].double().masked_fill(late, math.inf), descending=True, stable=True)
            kept = rank[:m].sort().values
            src = kept[kept >= m]
            holes = torch.ones(m, dtype=torch.bool, device=DEV)
            holes[kept[kept < m]] = False
            dst = holes.nonzero()[:, 0]
            score[b, h, dst], pos[b, h, dst] = score[b, h, src], pos[b, h, src]
            for x in (k, v):
                x[s["table"][b, dst // ps].long(), dst % ps, h] = x[s["table"][b, src // ps].long(), src % ps, h]
        score[b, :, m:], pos[b, :, m:] = 0.0, -1
    return dict(score=score, pos=pos, n=torch.tensor(new_n, dtype=torch.int32, device=DEV), k=k, v=v)


def _exact_verify(s):
    c = s["case"]
    accept, token = [], []
    for b in range(c["B"]):
        n = c["L"] if s["draft_len"] is None else int(s["draft_len"][b])
        a = 0
        while a < n:
            x = int(s["tok"][b, a])
            if not float(s["u"][b, a]) * float(s["draft"][b, a, x]) < float(s["target"][b, a, x]):
                break
            a += 1
        p = s["target"][b, a].double()
        w = (p - s["draft"][b, a].double()).clamp(min=0.0) if a < n else p
        w = w if bool((w > 0).any()) else p
        r = torch.where(w > 0, w / s["noise"][b].double(), torch.zeros_like(w))
        accept.append(a)
        token.append(int((r == r.max()).nonzero()[0, 0]) if float(r.max()) > 0 else -1)
    return dict(accept=torch.tensor(accept, dtype=torch.int32, device=DEV),
                token=torch.tensor(token, dtype=torch.int32, device=DEV))
