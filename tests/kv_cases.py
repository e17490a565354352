"""Blocks of queries on paged caches for the tests of attention and eviction."""
import numpy as np
import torch

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}    # unit roundoff: 8 and 11 significant bits
MASKS = ("none", "causal", "mixed", "random", "hidden")


def block_mask(kind, B, L, rng):
    """[B, L] words: bit t of row i lets position i see position t."""
    if kind == "none":
        return None
    full = (1 << L) - 1
    words = np.zeros((B, L), dtype=np.uint64)
    for b in range(B):
        for i in range(L):
            if kind == "causal" or (kind == "mixed" and i < (L + 1) // 2):
                words[b, i] = (1 << (i + 1)) - 1
            elif kind == "mixed":
                words[b, i] = full
            elif kind == "random":
                words[b, i] = int(rng.integers(0, 1 << 63)) & full
    return words                                  # "hidden": no row sees its block


class Case:
    """Random pages, block table, lengths and queries; ``junk`` fills every
    place that no sequence holds."""

    def __init__(self, B, L, H, Hkv, D, prefix, lens, mask="none", page=16, layout="nhd", dtype="bf16", seed=0,
                 q_std=2.0, junk=float("nan"), spare_pages=2):
        rng = np.random.default_rng(seed)
        dt = TYPES[dtype]
        self.B, self.L, self.H, self.Hkv, self.D, self.page, self.dtype = B, L, H, Hkv, D, page, dtype
        self.lens = list(lens)
        assert len(self.lens) == B
        need = [-(-n // page) for n in self.lens]
        cols = max(1, max(need))
        n_pages = sum(need) + spare_pages
        order = rng.permutation(n_pages)
        self.table = np.full((B, cols), 1 << 30, dtype=np.int32)     # past a sequence's pages: any id
        at = 0
        for b in range(B):
            self.table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
        shape = (n_pages, page, Hkv, D)
        k, v = (torch.from_numpy(rng.standard_normal(shape)).to(dt) for _ in range(2))
        held = torch.zeros(n_pages, page, dtype=torch.bool)
        for b, n in enumerate(self.lens):
            for j in range(n):
                held[self.table[b, j // page], j % page] = True
        for x in (k, v):
            x[~held] = junk
        self.k, self.v = k, v
        self.mask = block_mask(mask, B, L, rng)
        self.q = torch.from_numpy(q_std * rng.standard_normal((B, L, H, D))).to(dt)
        self.prefix = None
        if prefix is not None:
            self.prefix = tuple(torch.from_numpy(rng.standard_normal((prefix, Hkv, D))).to(dt) for _ in range(2))
        self.layout = layout
        self.scale = D ** -0.5
        self.rng = rng

    def own(self, x):
        import oracle.attention_oracle as ao
        pages = x.double().numpy()
        return [ao.own_rows(pages, self.table[b], n, self.page) for b, n in enumerate(self.lens)]

    def _laid(self, t, axes):
        return t.transpose(*axes).contiguous().cuda().transpose(*axes) if self.layout == "hnd" else t.cuda()

    def cache(self, brisk):
        return brisk.KVCache(self._laid(self.k, (1, 2)), self._laid(self.v, (1, 2)),
                             torch.from_numpy(self.table).cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda())

    def gpu_prefix(self):
        return None if self.prefix is None else tuple(self._laid(t, (0, 1)) for t in self.prefix)

    def gpu_mask(self):
        return None if self.mask is None else torch.from_numpy(self.mask.view(np.int64)).cuda()

    def oracle_prefix(self):
        return None if self.prefix is None or not len(self.prefix[0]) else tuple(t.double().numpy() for t in self.prefix)

    def attention(self):
        import oracle.attention_oracle as ao
        return ao.block_attention(self.q.double().numpy(), self.own(self.k), self.own(self.v), self.oracle_prefix(),
                                  self.mask, self.scale)
