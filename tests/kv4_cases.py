"""Caches held in 4 bits for the tests of writing, reading and attention."""
import numpy as np
import torch

import oracle.attention_oracle as ao
import oracle.kv4_oracle as k4
from kv_cases import TYPES, UNIT, block_mask

LEAST = {"bf16": 2.0 ** -126, "f16": 0.0}        # steps below the normal numbers of bf16 count as 0


def rounder(dtype):
    return lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(TYPES[dtype]).double().numpy()


def hold(x, dtype):
    return k4.hold(x.double().numpy(), rounder(dtype), LEAST[dtype])


def read_back(x, dtype):
    """What kv4_read gives for tokens x (a CPU tensor): type(fl(z + s c))."""
    z, s, c = hold(x, dtype)
    return torch.from_numpy((z + s * c).astype(np.float32)).to(TYPES[dtype])


def pages_for(brisk, n_pages, Hkv, D, page, fill=0xFF):
    """Pages whose places hold NaN heads until they are written."""
    return torch.full((n_pages, Hkv, brisk.kv4_page_bytes(page, D)), fill, dtype=torch.uint8, device="cuda")


class Case4:
    """Random tokens of sequences of ``lens`` in pages in no order, and a block's queries."""

    def __init__(self, brisk, B, L, H, Hkv, D, prefix, lens, mask="none", page=16, dtype="bf16", seed=0, q_std=1.0,
                 spare_pages=2, k=None, v=None, fill=0xFF):
        rng = np.random.default_rng(seed)
        dt = TYPES[dtype]
        self.B, self.L, self.H, self.Hkv, self.D, self.page, self.dtype = B, L, H, Hkv, D, page, dtype
        self.lens, self.scale = list(lens), D ** -0.5
        need = [-(-n // page) for n in lens]
        cols, n_pages = max(1, max(need)), sum(need) + spare_pages
        order = rng.permutation(n_pages)
        self.table = np.full((B, cols), 1 << 30, dtype=np.int32)
        at = 0
        for b in range(B):
            self.table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
        most = max(1, max(lens))
        channel = np.exp(0.5 * rng.standard_normal((Hkv, D)))
        mk = lambda c: torch.from_numpy((rng.standard_normal((B, most, Hkv, D)) + 0.3) * c).to(dt)  # noqa: E731
        self.k, self.v = (mk(channel) if k is None else k), (mk(1.0) if v is None else v)
        self.mask = block_mask(mask, B, L, rng)
        self.q = torch.from_numpy(q_std * rng.standard_normal((B, L, H, D))).to(dt)
        self.prefix = None
        if prefix is not None:
            self.prefix = tuple(torch.from_numpy(rng.standard_normal((prefix, Hkv, D))).to(dt) for _ in range(2))
        self.pages = pages_for(brisk, n_pages, Hkv, D, page, fill)
        self.seq_len = torch.tensor(self.lens, dtype=torch.int32).cuda()
        self.cache = brisk.KVCache4(self.pages, torch.from_numpy(self.table).cuda(), self.seq_len, D, dt)
        brisk.kv4_write(self.k.cuda(), self.v.cuda(), self.cache, torch.zeros(B, dtype=torch.int32, device="cuda"),
                        count=self.seq_len)

    def gpu_mask(self):
        return None if self.mask is None else torch.from_numpy(self.mask.view(np.int64)).cuda()

    def gpu_prefix(self):
        return None if self.prefix is None else tuple(t.cuda() for t in self.prefix)

    def expect(self):
        """out, lse and their tolerances.  With u the unit roundoff of the cache's type: the output's own
        rounding gives u |out|, that of a weight p s where it meets the codes u p s c; the fp32
        exponentials, sums and rescaling 2^-15 of the same sums, with 16 s for the codes and the
        number that bf16 codes stand on.  A logit's products and the sum of q are off by less than
        2^-18 scale sum |q| (|z| + 31 s), which moves every weight by that factor, and the
        log-sum-exp by that amount.  Prefix keys count as z alone."""
        B, L, H, D, G = self.B, self.L, self.H, self.D, self.H // self.Hkv
        u, q = UNIT[self.dtype], self.q.double().numpy()
        hk, hv = hold(self.k, self.dtype), hold(self.v, self.dtype)
        out, tol = np.zeros((B, L, H, D)), np.zeros((B, L, H, D))
        lse, ltol = np.full((B, L, H), -np.inf), np.zeros((B, L, H))
        for b, n in enumerate(self.lens):
            for i in range(L):
                vis = ao.sees(n, L, i, None if self.mask is None else self.mask[b, i])
                for h in range(H):
                    own = [[np.broadcast_to(y[b, :n, h // G][vis], (vis.sum(), D)) for y in x] for x in (hk, hv)]
                    if self.prefix is not None and len(self.prefix[0]):
                        pre = [x[:, h // G].double().numpy() for x in self.prefix]
                        own = [[np.concatenate([p if j == 0 else np.zeros_like(p), y]) for j, y in enumerate(x)]
                               for p, x in zip(pre, own)]
                    keys, values = own
                    if not len(keys[0]):
                        continue
                    z = self.scale * ((keys[0] + keys[1] * keys[2]) @ q[b, i, h])
                    m = z.max()
                    p = np.exp(z - m)
                    lse[b, i, h] = m + np.log(p.sum())
                    p /= p.sum()
                    out[b, i, h] = p @ (values[0] + values[1] * values[2])
                    logit, coded, fine = k4.scales(q[b, i, h], [y.max(1, keepdims=True) if j == 1 else y for j, y in enumerate(keys)],
                                                   values, p, self.scale)
                    d = 2.0 ** -18 * logit
                    tol[b, i, h] = u * (np.abs(out[b, i, h]) + coded) + (2.0 ** -15 + 2 * d) * fine + 2.0 ** -24
                    ltol[b, i, h] = d + 2.0 ** -20 * (1 + abs(lse[b, i, h]))
        return out, lse, tol, ltol

    def check(self, out, lse, want=None):
        o, z, tol, ltol = self.expect() if want is None else want
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        empty = z == -np.inf
        assert np.array_equal(lse == -np.inf, empty)
        assert (out[empty] == 0).all()
        assert (np.abs(out - o) <= tol).all(), np.nanmax(np.abs(out - o) / tol)
        assert (np.abs(lse - z)[~empty] <= ltol[~empty]).all(), np.nanmax((np.abs(lse - z)[~empty] / ltol[~empty]))
