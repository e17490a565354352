"""GPU checks of brisk_kv4_write at the largest steps that bf16 has: their reciprocal's second part
is a subnormal number, and codes are those of the definition all the same."""
import numpy as np
import pytest
import torch

import oracle.kv4_oracle as k4
from kv4_cases import LEAST, pages_for, read_back, rounder

pytestmark = pytest.mark.gpu

brisk = pytest.importorskip("paper_2609_33390_amd")
D = 64


def _bf16(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float64)).to(torch.bfloat16)


def _heads(rng, n, exponent):
    """Heads of steps of that exponent: elements at the middle between two codes, one ulp of bf16 beside it, and numbers
    so small that with z = -(c + 1/2) s they move a quotient by its last bit."""
    rows = []
    for _ in range(n):
        s = 2.0 ** exponent * (1 + rng.integers(0, 128) / 128)
        z = -s * rng.integers(1, 16) / 2
        x = _bf16(z + s * rng.integers(0, 31, D) / 2)
        x = (x.view(torch.int16) + torch.from_numpy(rng.integers(-1, 2, D)).to(torch.int16) * (x != 0)).view(torch.bfloat16)
        small = s * 2.0 ** -rng.integers(20, 27, D // 2) * rng.choice([-1, 1], D // 2) * (1 + rng.integers(0, 128, D // 2) / 128)
        x[torch.from_numpy(rng.choice(D, D // 2, replace=False))] = _bf16(small)
        x[0], x[1] = _bf16([z, z + (15 if exponent < 123 else 14) * s])
        rows.append(x)
    return torch.stack(rows)


def _check(k):
    """k [n, D], n a multiple of 64, as keys and, the other way round, as values."""
    k = k.view(1, -1, 4, D)
    v, T = k.flip(-1).contiguous(), k.shape[1]
    table = torch.arange(T // 16, dtype=torch.int32, device="cuda").view(1, -1)
    n = torch.tensor([T], dtype=torch.int32, device="cuda")
    cache = brisk.KVCache4(pages_for(brisk, T // 16, 4, D, 16), table, n, D)
    brisk.kv4_write(k.cuda(), v.cuda(), cache, n - T)
    rk, rv = brisk.kv4_read(cache, T)
    for x, y in ((k, rk.cpu()), (v, rv.cpu())):
        want = read_back(x, "bf16")
        assert torch.isfinite(want).all()
        assert torch.equal(y, want), (y != want).sum()


@pytest.mark.parametrize("exponent", [60, 63, 64, 65, 90, 103, 110, 116, 119, 120, 121, 122, 123])
def test_codes_of_large_steps(exponent):
    _check(_heads(np.random.default_rng(exponent), 2048, exponent))


def test_a_quotient_one_bit_past_the_middle():
    """s = 247/128 2^122, z = -s/2 and an element of 2^98: the quotient is 1/2 and its last bit, so code 1."""
    s = 247 / 128 * 2.0 ** 122
    x = _bf16([-s / 2, 2.0 ** 98, 14.5 * s] + [0.0] * (D - 3))
    z, step, c = k4.hold(x.double().numpy()[None], rounder("bf16"), LEAST["bf16"])
    assert step == s and c[0, :4].tolist() == [0, 1, 15, 0]
    _check(x.expand(64, D).contiguous())
