"""The decoding example: the attention, score, eviction and verification calls run together."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

pytest.importorskip("paper_2609_33390_amd")
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_example_decodes_within_its_budget():
    import block_decoding
    texts, accepted, lens = block_decoding.decode(rounds=20, B=3, L=8, prompt=70, budget=24, recent=8, seed=3)
    torch.cuda.synchronize()
    assert accepted.shape == (20, 3) and int(accepted.min()) >= 0 and int(accepted.max()) <= 7
    for b, t in enumerate(texts):
        assert len(t) == 1 + 20 + int(accepted[:, b].sum())       # the first anchor, then a token and the accepted a round
        assert all(0 <= x < 1003 for x in t)
        assert int(lens[b]) == min(24, 20 + int(accepted[:, b].sum()))


def test_example_repeats_itself():
    import block_decoding
    assert block_decoding.decode(rounds=5, seed=4)[0] == block_decoding.decode(rounds=5, seed=4)[0]
