"""Speculative block decoding on a shared prefix and a bounded cache.

Several sequences continue one long prompt.  Each round writes a block (the
last committed token and the drafts after it) to the paged cache and makes one
pass over it:

  block_attention  the block's rows over the shared prompt and each own cache
  draft_verify     the drafts against the pass's probabilities
  cache_score      the attention weight that the cached keys received
  cache_evict      back to the budget, when a cache has outgrown it

With ``bits=4`` the cache holds its keys and values in 4 bits instead, and all of
them: kv4_write and kv4_attention take the place of the copies and of
block_attention, and nothing is evicted.

The model is one attention layer with random weights (there is nothing to
download); what it decodes is noise, how it decodes is not.

    python examples/block_decoding.py [rounds] [bits]
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_33390_amd as brisk  # noqa: E402


class Layer:
    """Random weights of one attention layer, a language-model head and a draft head a position."""

    def __init__(self, d, H, Hkv, D, V, L, g):
        def w(*shape):
            return (torch.randn(*shape, generator=g, device="cuda") * shape[-1] ** -0.5).to(torch.bfloat16)

        self.H, self.Hkv, self.D, self.V = H, Hkv, D, V
        self.embed, self.qkv, self.out, self.head = w(V, d), w((H + 2 * Hkv) * D, d), w(d, H * D), w(V, d)
        self.draft = w(L - 1, d, d)

    def project(self, tokens):
        """Queries, keys and values of [..., n] tokens, heads split: views of one product."""
        x = (self.embed[tokens] @ self.qkv.T).unflatten(-1, (self.H + 2 * self.Hkv, self.D))
        return x[..., :self.H, :], x[..., self.H:self.H + self.Hkv, :], x[..., self.H + self.Hkv:, :]

    def finish(self, tokens, attended):
        return self.embed[tokens] + attended.flatten(-2) @ self.out.T

    def probs(self, hidden):
        return torch.softmax((hidden @ self.head.T).float() * 2.0, -1)


def decode(rounds=8, B=4, L=8, prompt=300, budget=64, recent=16, seed=0, bits=16):
    """Decodes ``rounds`` blocks; returns the committed tokens of each sequence,
    the accepted lengths [rounds, B] and the final cache lengths."""
    if bits == 4:
        return decode4(rounds, B, L, prompt, seed)[:3]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    layer = Layer(256, 8, 2, 32, 1003, L, g)
    page, slots = 16, (budget + L + 15) // 16 * 16
    pages = slots // page
    k_pages = torch.zeros(B * pages, page, layer.Hkv, layer.D, dtype=torch.bfloat16, device="cuda")
    v_pages = torch.zeros_like(k_pages)
    table = torch.arange(B * pages, dtype=torch.int32, device="cuda").view(B, pages)
    seq_len = torch.zeros(B, dtype=torch.int32, device="cuda")
    cache = brisk.KVCache(k_pages, v_pages, table, seq_len)
    _, pk, pv = layer.project(torch.randint(0, layer.V, (prompt,), generator=g, device="cuda"))

    score = torch.zeros(B, layer.Hkv, slots, device="cuda")
    pos = torch.full((B, layer.Hkv, slots), -1, dtype=torch.int32, device="cuda")
    next_pos = torch.full((B,), prompt, dtype=torch.int32, device="cuda")
    at = torch.arange(B, device="cuda")[:, None]
    place, slot = torch.arange(L, device="cuda"), torch.arange(slots, device="cuda")
    causal = torch.tensor([[(2 << i) - 1 for i in range(L)]], device="cuda").repeat(B, 1)

    anchor = torch.randint(0, layer.V, (B, 1), generator=g, device="cuda")
    law = torch.full((B, L - 1, layer.V), 1.0 / layer.V, device="cuda")
    committed, accepted = [anchor], []
    for _ in range(rounds):
        # drafts from their law, then the block into the cache behind what is committed
        drafts = (law / torch.empty_like(law).exponential_(generator=g)).argmax(-1)
        tokens = torch.cat([anchor, drafts], 1)
        q, k, v = layer.project(tokens)
        begin = seq_len.long()[:, None]
        into = table[at, (begin + place) // page].long(), (begin + place) % page
        k_pages[into], v_pages[into] = k, v
        pos.scatter_(2, (begin + place)[:, None].expand(-1, layer.Hkv, -1),
                     (next_pos[:, None] + place.int())[:, None].expand(-1, layer.Hkv, -1))
        seq_len += L

        attended, lse = brisk.block_attention(q, cache, prefix=(pk, pv), block_mask=causal)
        hidden = layer.finish(tokens, attended)
        u = torch.rand(B, L - 1, generator=g, device="cuda")
        noise = torch.empty(B, layer.V, device="cuda").exponential_(generator=g)
        a, token = brisk.draft_verify(layer.probs(hidden), law, drafts.int(), u, noise)
        brisk.cache_score(q, lse, cache, score, block_mask=causal, decay=0.9, out=score)

        # commit the anchor and the accepted drafts; what was rejected is forgotten
        seq_len -= (L - 1) - a
        next_pos += 1 + a
        score.masked_fill_(slot >= seq_len[:, None, None], 0.0)
        score, pos, kept = brisk.cache_evict(cache, score, pos, next_pos, budget, recent)
        seq_len.copy_(kept)

        anchor = token.long()[:, None]
        last = hidden[torch.arange(B, device="cuda"), a.long()]
        law = layer.probs(torch.stack([last @ m for m in layer.draft], 1))
        committed.append(torch.where(place[:L - 1] < a[:, None], drafts, -1))
        committed.append(anchor)
        accepted.append(a)
    out = torch.cat(committed, 1)
    return [row[row >= 0].tolist() for row in out], torch.stack(accepted).cpu(), seq_len.cpu()


def decode4(rounds=8, B=4, L=8, prompt=300, seed=0):
    """The same over a cache in 4 bits that keeps every token: what ``decode`` returns, the
    layer and the cache."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    layer = Layer(256, 8, 2, 32, 1003, L, g)
    page, pages = 16, -(-(rounds * L) // 16)
    pool = torch.zeros(B * pages, layer.Hkv, brisk.kv4_page_bytes(page, layer.D), dtype=torch.uint8, device="cuda")
    table = torch.randperm(B * pages, generator=g, device="cuda").to(torch.int32).view(B, pages)
    seq_len = torch.zeros(B, dtype=torch.int32, device="cuda")
    cache = brisk.KVCache4(pool, table, seq_len, layer.D)
    _, pk, pv = layer.project(torch.randint(0, layer.V, (prompt,), generator=g, device="cuda"))

    place = torch.arange(L, device="cuda")
    causal = torch.tensor([[(2 << i) - 1 for i in range(L)]], device="cuda").repeat(B, 1)
    anchor = torch.randint(0, layer.V, (B, 1), generator=g, device="cuda")
    law = torch.full((B, L - 1, layer.V), 1.0 / layer.V, device="cuda")
    committed, accepted = [anchor], []
    for _ in range(rounds):
        drafts = (law / torch.empty_like(law).exponential_(generator=g)).argmax(-1)
        tokens = torch.cat([anchor, drafts], 1)
        q, k, v = layer.project(tokens)
        brisk.kv4_write(k, v, cache, seq_len)      # behind what is committed
        seq_len += L

        attended, _ = brisk.kv4_attention(q, cache, prefix=(pk, pv), block_mask=causal)
        hidden = layer.finish(tokens, attended)
        u = torch.rand(B, L - 1, generator=g, device="cuda")
        noise = torch.empty(B, layer.V, device="cuda").exponential_(generator=g)
        a, token = brisk.draft_verify(layer.probs(hidden), law, drafts.int(), u, noise)
        seq_len -= (L - 1) - a                     # what was rejected is written over

        anchor = token.long()[:, None]
        last = hidden[torch.arange(B, device="cuda"), a.long()]
        law = layer.probs(torch.stack([last @ m for m in layer.draft], 1))
        committed.append(torch.where(place[:L - 1] < a[:, None], drafts, -1))
        committed.append(anchor)
        accepted.append(a)
    out = torch.cat(committed, 1)
    return [row[row >= 0].tolist() for row in out], torch.stack(accepted).cpu(), seq_len.cpu(), layer, cache


if __name__ == "__main__":
    n = int(sys.argv[1]) if len(sys.argv) > 1 else 8
    texts, acc, lens = decode(n, bits=int(sys.argv[2]) if len(sys.argv) > 2 else 16)
    for b, t in enumerate(texts):
        print(f"sequence {b}: {len(t)} tokens, accepted {acc[:, b].tolist()}, cache {int(lens[b])}: {t[:10]} ...")
