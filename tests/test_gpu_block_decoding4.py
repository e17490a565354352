"""The decoding loop of the example over a cache in 4 bits: that its lengths add up and
that the cache holds what was committed, nothing of what was rejected."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

brisk = pytest.importorskip("paper_2609_33390_amd")


@pytest.mark.parametrize("rounds,B,L", [(5, 4, 8), (7, 3, 5), (3, 1, 16)])
def test_cache_holds_the_committed_tokens(rounds, B, L):
    from block_decoding import decode, decode4
    from kv4_cases import read_back
    texts, acc, lens, layer, cache = decode4(rounds, B, L, prompt=70, seed=rounds)
    assert torch.equal(lens.long(), (acc.long() + 1).sum(0))
    k, v = brisk.kv4_read(cache, int(lens.max()))
    for b in range(B):
        n = int(lens[b])
        assert len(texts[b]) == n + 1              # the last token is not in the cache yet
        # the products of these rows may round otherwise in another batch: held values of the cache's own
        # rounding are compared where the row is the same
        _, wk, wv = layer.project(torch.tensor(texts[b][:n], device="cuda"))
        for x, y in ((wk, k), (wv, v)):
            want = read_back(x.cpu(), "bf16")
            step = (x.float().amax(-1) - x.float().amin(-1)).cpu() / 15
            assert ((y[b, :n].cpu().float() - want.float()).abs() <= 0.1 * step[..., None] + want.float().abs() * 2.0 ** -6).float().mean() > 0.99
        assert (k[b, n:] == 0).all()
    again = decode(rounds, B, L, prompt=70, seed=rounds, bits=4)
    assert again[0] == texts and torch.equal(again[1], acc) and torch.equal(again[2], lens)
