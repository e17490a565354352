"""GPU checks that keys and values which a row does not see have no effect on it, whatever their size: not on
the logit that it subtracts or the scale that its weights are held at either."""
import numpy as np
import pytest
import torch

from kv4_cases import Case4
from kv_cases import TYPES, UNIT

pytestmark = pytest.mark.gpu

brisk = pytest.importorskip("paper_2609_33390_amd")


def _run(c):
    print(f"[kv4 hidden] B={c.B} L={c.L} H={c.H}/{c.Hkv} D={c.D} lens={c.lens[:4]} {c.dtype}", flush=True)
    out, lse = brisk.kv4_attention(c.q.cuda(), c.cache, block_mask=c.gpu_mask(), scale=c.scale)
    torch.cuda.synchronize()
    return out, lse


def _huge(v, at, dtype):
    """The values of a slot as one of the largest step that the type has (one past the largest of fp32 would not be finite)."""
    v = v.clone()
    top = torch.finfo(TYPES[dtype]).max / (1 if dtype == "f16" else 4)
    v[:, at] = -top
    v[:, at, :, ::2] = top
    return v


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L,G,n", [(2, 1, 40), (2, 1, 3000), (2, 4, 700), (5, 2, 3000), (16, 1, 500), (20, 1, 300), (32, 4, 9000),
                                   (40, 2, 5000)])
def test_rows_are_the_same_bits_beside_any_hidden_value(L, G, n, D, dtype):
    """The block's last slot, which only its last position sees; bf16 values are small numbers beside it."""
    small = 2.0 ** -60 if dtype == "bf16" else 1.0
    g = torch.Generator().manual_seed(n)
    k = torch.randn(1, n, 2, D, generator=g).to(TYPES[dtype])
    v = (torch.randn(1, n, 2, D, generator=g) * small).to(TYPES[dtype])
    outs = []
    for x in (v, _huge(v, n - 1, dtype)):
        c = Case4(brisk, 1, L, 2 * G, 2, D, None, [n], mask="causal", dtype=dtype, seed=n + L, k=k, v=x)
        out, lse = _run(c)
        outs.append((out[:, :L - 1], lse[:, :L - 1], out[:, L - 1]))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    assert torch.isfinite(outs[1][2]).all() and (outs[1][2] != outs[0][2]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("L", [2, 20, 40])
def test_rows_without_keys_beside_hidden_values(L, dtype):
    """Blocks that are all there is, seen by the last position alone: the rows before it are empty."""
    g = torch.Generator().manual_seed(L)
    k, v = (torch.randn(1, L, 2, 64, generator=g).to(TYPES[dtype]) for _ in range(2))
    for x in (v, _huge(v, L // 2, dtype)):
        c = Case4(brisk, 1, L, 4, 2, 64, None, [L], mask="causal", dtype=dtype, seed=L, k=k, v=x)
        c.mask[:, :L - 1] = 0
        out, lse = _run(c)
        c.check(out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("L", [2, 20])
def test_weak_keys_count_beside_a_hidden_value(L, dtype):
    """One key of weight 1 and value 0 among 40000 of weight 2^-20, and a hidden slot of the largest values.  The
    tolerance: a rounding of each weight and of the output, the subtracted logit's own, and the exponentials'."""
    dt, n, D = TYPES[dtype], 40000, 64
    k, v = torch.zeros(1, n, 1, D, dtype=dt), torch.ones(1, n, 1, D, dtype=dt)
    v[..., 1::2] = 0.5
    k[:, n // 3, 0, 0] = 15.0                        # of a step of 1: held as it is
    v[:, n // 3] = 0.0
    c = Case4(brisk, 1, L, 1, 1, D, None, [n], mask="causal", dtype=dtype, k=k, v=_huge(v, n - 1, dtype), page=64)
    c.q.zero_()
    c.q[..., 0] = 1.0
    c.scale = 20 * np.log(2.0) / 15
    out = _run(c)[0][0, :L - 1, 0].double().cpu().numpy()
    weak = np.array([n - 1 - (L - 1 - i) for i in range(L - 1)]) * 2.0 ** -20
    weak = (weak / (1 + weak))[:, None]
    assert (np.abs(out[:, 0::2] - weak) <= 3 * UNIT[dtype] * weak + 2.0 ** -20).all()
    assert (np.abs(out[:, 1::2] - weak / 2) <= 3 * UNIT[dtype] * weak + 2.0 ** -20).all()


def test_f16_weights_beside_a_seen_value_of_a_large_step():
    """A key of weight 2^-40 whose value's step is the largest there is: weights times steps are then held in steps of
    2^-36 of it, each off by half of that, for codes of at most 8 from the middle."""
    n, D = 2000, 64
    g = torch.Generator().manual_seed(2)
    k, v = torch.zeros(1, n, 1, D, dtype=torch.float16), torch.randn(1, n, 1, D, generator=g).to(torch.float16)
    k[:, 5, 0, 0] = -15.0
    v = _huge(v, 5, "f16")
    c = Case4(brisk, 1, 1, 1, 1, D, None, [n], dtype="f16", k=k, v=v)
    c.q.zero_()
    c.q[..., 0] = 1.0
    c.scale = 40 * np.log(2.0) / 15
    o, z, tol, ltol = c.expect()
    step = 2 * torch.finfo(torch.float16).max / 15
    c.check(*_run(c), want=(o, z, tol + 8 * 2.0 ** -36 * step, ltol))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("size", [20.0, 1e4])
@pytest.mark.parametrize("L,G,n", [(2, 1, 40), (2, 4, 700), (5, 2, 3000), (16, 1, 500), (20, 1, 300), (32, 4, 9000), (40, 2, 5000)])
def test_rows_are_the_same_bits_beside_any_hidden_key(L, G, n, size, D, dtype):
    """The block's last slot, which only its last position sees, has a key whose logits are far above all others (or so
    large that differences of them are taken before they are scaled): no other row's maximum moves with that one's."""
    g = torch.Generator().manual_seed(n)
    k, v = (torch.randn(1, n, 2, D, generator=g).to(TYPES[dtype]) for _ in range(2))
    q = torch.randn(1, L, 2 * G, D, generator=g).to(TYPES[dtype])
    q[:, L - 1] = q[:, L - 1, :1]
    far = k.clone()
    far[0, n - 1] = (size * q[0, L - 1, 0].float()).to(TYPES[dtype])
    outs = []
    for x in (k, far):
        c = Case4(brisk, 1, L, 2 * G, 2, D, None, [n], mask="causal", dtype=dtype, seed=n + L, k=x, v=v)
        c.q = q                                    # logits so alike that the subtracted one may lag behind the largest
        out, lse = _run(c)
        outs.append((out[:, :L - 1], lse[:, :L - 1], lse[:, L - 1]))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    assert torch.isfinite(outs[1][2]).all() and (outs[1][2] > outs[0][2] + 100).all()
