"""Host-side checks of what the attention over the 4-bit cache runs on: that the calls of the GPU
tests still take every kernel there is (no GPU needed)."""
import itertools

import pytest

from kv4_plan import plan4
from kv4_plan_cases import CASES, HEADS, LONG, LONG_RUNS

# rows of a tile, wavefronts, lanes that share a row
KERNELS = {(16, waves, lanes) for waves in (2, 4, 8) for lanes in (1, 2, 4)} | {(32, 4, 1), (64, 4, 1)}


def _plans():
    """Of every case: the kernel, its plan, rows of a key head, steps of the first wavefront, whether there is a prefix."""
    for B, L, G, Hkv, n, prefix, _ in CASES:
        p = plan4(B, L, G * Hkv, Hkv, HEADS[0], prefix, _bound(n))
        yield (p.rows, p.waves, p.lanes), p, L * G, -(-min(p.run, n) // (32 * p.waves)), prefix > 0


def _bound(n):
    return -(-n // 64) * 64                        # the binding's: what the table addresses, in pages of 64


@pytest.mark.parametrize("kind", ["any", "several runs", "by length", "32 steps"])
def test_every_kernel_is_taken(kind):
    seen = {k for k, p, _, steps, _ in _plans()
            if kind == "any" or kind == "several runs" and p.runs > 1 or kind == "by length" and p.by_length or kind == "32 steps" and steps >= 32}
    assert seen == KERNELS, KERNELS - seen


@pytest.mark.parametrize("tile", [32, 64])
def test_tiles_of_many_rows(tile):
    """Several tiles, the last one not full, with a prefix and without, and a single one."""
    of = [(p.tiles, rows % tile, prefix) for k, p, rows, _, prefix in _plans() if k[0] == tile]
    assert {(tiles > 1, rest != 0, prefix) for tiles, rest, prefix in of} >= {(True, True, True), (True, True, False)}
    assert any(tiles == 1 for tiles, _, _ in of)


@pytest.mark.parametrize("D", range(8, 136, 8))
def test_both_widths(D):
    assert plan4(1, 1, 4, 1, D, 0, 100).width == (64 if D <= 64 else 128)
    assert {plan4(1, 1, 4, 1, d, 0, 100).width for d in HEADS} == {64, 128}


@pytest.mark.parametrize("B", [1, 3, 64, 65, 256])
@pytest.mark.parametrize("n", [0, 1, 500, 33000])
def test_plans_are_launches_that_there_are(B, n):
    """One of the kernels, whole steps a run, and runs that cover the bound, the last one not empty."""
    for L, G, Hkv in itertools.product((1, 2, 4, 7, 17, 33, 64), (1, 3, 5, 16), (1, 8)):
        p = plan4(B, L, G * Hkv, Hkv, 64, 0, n)
        assert (p.rows, p.waves, p.lanes) in KERNELS
        assert p.rows * p.tiles >= L * G > p.rows * (p.tiles - 1)
        assert p.run % (32 * p.waves) == 0 and p.run * p.runs >= n and (p.runs == 1 or p.run * (p.runs - 1) < n)
        assert p.rows > 16 or p.lanes * L * G <= 16
        assert not p.by_length or 1 < B <= 64


def test_no_own_keys_no_launch():
    assert plan4(2, 4, 8, 2, 64, 100, 0) is None


@pytest.mark.parametrize("B,L,G,Hkv,rows,waves", LONG_RUNS)
def test_long_runs_are_not_split(B, L, G, Hkv, rows, waves):
    p = plan4(B, L, G * Hkv, Hkv, 64, 0, LONG)
    assert (p.rows, p.waves, p.runs, p.run) == (rows, waves, 1, LONG)
