"""Calls that take every kernel of the attention over the 4-bit cache, and their expected results."""
import numpy as np
import torch

from kv4_cases import hold, pages_for
from kv_cases import TYPES, UNIT, block_mask

# B, L, query heads a key head, key heads, slots of the longest cache, prefix, mask
CASES = [
    # two wavefronts: whole caches, batches by length, runs, and 32 steps and more of a wavefront
    (6, 1, 3, 2, 100, 0, "none"), (6, 5, 1, 2, 100, 50, "causal"), (6, 3, 4, 2, 60, 50, "random"),
    (40, 1, 3, 32, 70, 0, "none"), (40, 5, 1, 32, 70, 0, "causal"), (40, 3, 3, 32, 40, 0, "hidden"),
    (1, 1, 3, 1, 2000, 0, "none"), (1, 1, 7, 1, 2000, 40, "none"), (1, 3, 3, 1, 2000, 0, "causal"),
    (256, 1, 4, 4, 2048, 0, "none"), (256, 1, 7, 4, 2048, 0, "none"), (256, 1, 12, 4, 2048, 0, "none"),
    # four
    (6, 1, 3, 2, 400, 0, "none"), (6, 1, 7, 2, 400, 0, "none"), (6, 4, 4, 1, 300, 0, "causal"),
    (40, 1, 2, 16, 512, 0, "none"), (40, 2, 3, 16, 512, 0, "mixed"), (40, 4, 3, 16, 500, 0, "causal"),
    (1, 1, 2, 1, 16000, 0, "none"), (1, 2, 4, 1, 16000, 0, "causal"), (1, 4, 4, 1, 16000, 20, "causal"),
    (256, 1, 4, 2, 4200, 0, "none"), (256, 1, 7, 2, 4200, 0, "none"), (256, 1, 12, 2, 4200, 0, "none"),
    # eight
    (6, 1, 4, 2, 700, 0, "none"), (6, 1, 8, 2, 700, 0, "none"), (6, 4, 4, 2, 700, 0, "causal"),
    (40, 1, 2, 8, 1000, 0, "none"), (40, 2, 4, 8, 1000, 0, "causal"), (40, 4, 4, 8, 1000, 0, "mixed"),
    (1, 1, 2, 1, 32000, 0, "none"), (1, 2, 4, 1, 32000, 0, "causal"), (1, 16, 1, 1, 32000, 0, "causal"),
    (256, 1, 4, 1, 8300, 0, "none"), (256, 1, 7, 1, 8300, 0, "none"), (128, 1, 12, 1, 16400, 0, "none"),
    (64, 4, 4, 8, 4096, 0, "causal"),
    # tiles of 32 rows: one, several, the last one not full, with a prefix, in runs, 33 steps
    (6, 17, 1, 2, 70, 0, "causal"), (6, 9, 3, 2, 300, 40, "causal"), (1, 17, 2, 1, 1000, 0, "mixed"),
    (40, 11, 3, 8, 100, 0, "causal"), (3, 23, 3, 2, 200, 30, "causal"), (3, 32, 5, 2, 300, 0, "random"), (64, 16, 2, 8, 4200, 0, "causal"),
    # tiles of 64 rows: the same
    (48, 33, 1, 16, 100, 33, "causal"), (128, 40, 5, 1, 130, 40, "mixed"), (8, 33, 3, 32, 64, 40, "random"),
    (12, 50, 2, 32, 64, 40, "causal"), (1, 33, 5, 8, 20000, 0, "causal"), (1, 35, 5, 8, 20000, 40, "mixed"),
    (1, 50, 8, 16, 20000, 0, "causal"),
]
HEADS = (64, 128)                                  # one of each width


class PlanCase:
    """A batch made of a few sequences, each of them several times and in no order."""

    def __init__(self, brisk, B, L, G, Hkv, n, prefix, mask, D, dtype, page=64):
        rng = np.random.default_rng(B + 64 * L + n)
        g = torch.Generator().manual_seed(n + L)
        dt, self.dtype, self.G, self.L, self.scale = TYPES[dtype], dtype, G, L, D ** -0.5
        self.lens = [n, n - n // 3, min(n, 33), 1, 0][:B]
        P = len(self.lens)
        self.which = np.concatenate([np.arange(P), rng.integers(0, P, B - P)])
        rng.shuffle(self.which[1:])
        self.k, self.v = (torch.randn(P, n, Hkv, D, generator=g).to(dt) for _ in range(2))
        self.q = torch.randn(P, L, G * Hkv, D, generator=g).to(dt)
        self.prefix = tuple(torch.randn(prefix, Hkv, D, generator=g).to(dt) for _ in range(2)) if prefix else None
        self.mask = block_mask(mask, P, L, rng)
        cols = -(-n // page)
        pages = pages_for(brisk, P * cols, Hkv, D, page)
        table = torch.from_numpy(rng.permutation(P * cols).astype(np.int32).reshape(P, cols)).cuda()
        lens = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        brisk.kv4_write(self.k.cuda(), self.v.cuda(), brisk.KVCache4(pages, table, lens, D, dt), torch.zeros_like(lens), count=lens)
        at = torch.from_numpy(self.which).cuda()
        self.cache = brisk.KVCache4(pages, table[at].contiguous(), lens[at].contiguous(), D, dt)
        self.gpu_q = self.q.cuda()[at].contiguous()
        self.gpu_mask = None if self.mask is None else torch.from_numpy(self.mask.view(np.int64)).cuda()[at].contiguous()

    def expect(self, s, h):
        """out, lse and tolerances [L, G(, D)] of sequence s and key head h, the tolerances as in kv4_cases.Case4."""
        u, n, L = UNIT[self.dtype], self.lens[s], self.L
        (zk, sk, ck), (zv, sv, cv) = (hold(x[s, :n, h], self.dtype) for x in (self.k, self.v))
        key, size, value, coded, fine = zk + sk * ck, (np.abs(zk) + 31 * sk).max(-1), zv + sv * cv, np.abs(zv) + sv * cv, np.abs(zv) + 16 * sv
        fine = np.broadcast_to(fine, value.shape)
        sees = np.ones((L, n), dtype=bool)
        if self.mask is not None:
            for t in range(L):
                if n - L + t >= 0:
                    sees[:, n - L + t] = [(int(w) >> t) & 1 for w in self.mask[s]]
        if self.prefix is not None:
            pk, pv = (x[:, h].double().numpy() for x in self.prefix)
            key, size = np.concatenate([pk, key]), np.concatenate([np.abs(pk).max(-1), size])
            value, coded, fine = (np.concatenate([a, b]) for a, b in ((pv, value), (np.abs(pv), coded), (np.abs(pv), fine)))
            sees = np.concatenate([np.ones((L, len(pk)), dtype=bool), sees], 1)
        q = self.q[s, :, h * self.G:(h + 1) * self.G].double().numpy()
        out, tol = np.zeros(q.shape), np.zeros(q.shape)
        lse, ltol = np.full(q.shape[:2], -np.inf), np.zeros(q.shape[:2])
        for i in range(L):
            if not sees[i].any():
                continue
            z = self.scale * (q[i] @ key[sees[i]].T)
            m = z.max(1, keepdims=True)
            p = np.exp(z - m)
            lse[i] = m[:, 0] + np.log(p.sum(1))
            p /= p.sum(1, keepdims=True)
            out[i] = p @ value[sees[i]]
            d = 2.0 ** -18 * self.scale * np.abs(q[i]).sum(1) * size[sees[i]].max()
            tol[i] = u * (np.abs(out[i]) + p @ coded[sees[i]]) + (2.0 ** -15 + 2 * d[:, None]) * (p @ fine[sees[i]]) + 2.0 ** -24
            ltol[i] = d + 2.0 ** -20 * (1 + np.abs(lse[i]))
        return out, lse, tol, ltol

    def check(self, out, lse):
        """Each sequence against the definition, and its copies: the same bits, but over a prefix, whose tiles hold rows
        of several sequences (one that needs a larger logit subtracted moves that of the others at the same step)."""
        P, Hkv = len(self.lens), self.k.shape[2]
        first = torch.tensor([int(np.argmax(self.which == s)) for s in range(P)], device="cuda")
        at = first[torch.from_numpy(self.which).cuda()]
        if self.prefix is None:
            assert torch.equal(out[at], out) and torch.equal(lse[at], lse)
        for s in range(P):
            copies = first[s:s + 1] if self.prefix is None else torch.from_numpy(np.flatnonzero(self.which == s)).cuda()
            for h in {0, Hkv - 1}:
                o, z, tol, ltol = self.expect(s, h)
                got, l = (x[copies, :, h * self.G:(h + 1) * self.G].double().cpu().numpy() for x in (out, lse))
                empty = z == -np.inf
                assert ((l == -np.inf) == empty).all() and (got[:, empty] == 0).all(), (s, h)
                assert (np.abs(got - o) <= tol).all(), (s, h, np.nanmax(np.abs(got - o) / tol))
                assert (np.abs(l[:, ~empty] - z[~empty]) <= ltol[~empty]).all(), (s, h)


# Batches that fill the GPU with whole caches: one run of 131072 slots, which takes a wavefront up to 65536 of them.  B, L,
# query heads a key head, key heads; rows of a tile and wavefronts
LONG_RUNS = [(64, 1, 4, 32, 16, 2), (64, 1, 16, 16, 16, 4), (64, 1, 16, 8, 16, 8), (64, 16, 2, 16, 32, 4), (64, 16, 4, 16, 64, 4)]
LONG = 131072
