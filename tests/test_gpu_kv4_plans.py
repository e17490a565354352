"""GPU checks of brisk_kv4_attention on every kernel that it dispatches to, against the definition in 64
bits.  Which kernels these calls take is asserted without a GPU, in test_kv4_plan_cpu."""
import numpy as np
import pytest
import torch

from kv4_cases import hold, pages_for
from kv4_plan_cases import CASES, HEADS, LONG, LONG_RUNS, PlanCase
from kv_cases import TYPES

pytestmark = pytest.mark.gpu

brisk = pytest.importorskip("paper_2609_33390_amd")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", HEADS)
@pytest.mark.parametrize("case", CASES, ids=str)
def test_every_kernel(case, D, dtype):
    print(f"[kv4 plans] {case} D={D} {dtype}", flush=True)
    c = PlanCase(brisk, *case, D, dtype)
    out, lse = brisk.kv4_attention(c.gpu_q, c.cache, prefix=None if c.prefix is None else tuple(x.cuda() for x in c.prefix),
                                   block_mask=c.gpu_mask, scale=c.scale)
    torch.cuda.synchronize()
    c.check(out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("B,L,G,Hkv,rows,waves", LONG_RUNS)
def test_sums_of_one_long_run(B, L, G, Hkv, rows, waves, dtype):
    """131072 slots and weights that differ little, all sequences over the same cache; 16 rows of key head 0, 1024 outputs.
    The error's squares are at most those of independent roundings: of the output, u / sqrt(3) of itself in the mean
    square; of each weight times its step r, the same of it times the code's distance from 8; and of the fp32 sums, one unit
    in the last place for each step of 32 slots.  Those sums are of codes on 64 (f16) or 128 (bf16), with the 8, and are
    brought back to the middle after 31 steps, so they grow from about 0 to A = 31 * 32 * (72 or 136) of a mean weight times
    step, in the mean square A / sqrt(3).  A fifth more, since 1024 squares' sum is known to 5 percent."""
    dt, D, page, n = TYPES[dtype], 64, 256, LONG
    u = torch.finfo(dt).eps / 2
    g = torch.Generator(device="cuda").manual_seed(B + G)
    k, v = (torch.randn(1, n, Hkv, D, generator=g, device="cuda", dtype=dt) for _ in range(2))
    q = (0.3 * torch.randn(B, L, G * Hkv, D, generator=g, device="cuda")).to(dt)
    pages = pages_for(brisk, n // page, Hkv, D, page)
    table = torch.randperm(n // page, generator=g, device="cuda").to(torch.int32).view(1, -1)
    lens = torch.full((B,), n, dtype=torch.int32, device="cuda")
    brisk.kv4_write(k, v, brisk.KVCache4(pages, table, lens[:1], D, dt), lens[:1] - n)
    out = brisk.kv4_attention(q, brisk.KVCache4(pages, table.expand(B, -1).contiguous(), lens, D, dt))[0]
    of = lambda x: x[:, :, :G].reshape(-1, D)[:16].double().cpu().numpy()                       # noqa: E731
    (z, s, a), (y, r, d) = ([np.broadcast_to(x, (n, D)) for x in hold(t[0, :, 0].cpu(), dtype)] for t in (k, v))
    p = of(q) @ (z + s * a).T * D ** -0.5
    p = np.exp(p - p.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    want = p @ (y + r * d)
    sums = 31 * 32 * (72 if dtype == "f16" else 136) * r.mean() / n
    fine = (n / 32) * (2.0 ** -23 * sums) ** 2 / 9 * want.size
    rounded = u * u / 3 * ((want ** 2).sum() + ((p ** 2) @ ((r * (d - 8)) ** 2)).sum())
    off = ((of(out) - want) ** 2).sum()
    print(f"[kv4 long run] {off ** 0.5 / (want ** 2).sum() ** 0.5:.2e} of {((fine + rounded) / (want ** 2).sum()) ** 0.5:.2e}", flush=True)
    assert off <= 1.2 * (fine + rounded)
