"""Oracle of the cache held in 4 bits: how a head of keys or values is held, in
64 bits but for the roundings that the definition has."""
from __future__ import annotations

import numpy as np


def hold(x, round_to, least_step):
    """(z, s, c) of heads x [..., D] float64: z lowest value, s step, c codes.

    ``round_to`` rounds a float64 array to the cache's type (nearest even);
    steps below ``least_step`` count as 0."""
    with np.errstate(invalid="ignore", over="ignore"):
        z, top = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
        span = (top - z).astype(np.float32)
        bad = ~np.isfinite(x).all(-1, keepdims=True) | ~np.isfinite(span)
        s = round_to((span / np.float32(15)).astype(np.float64))
    s = np.where(bad | (s < least_step), 0.0, s)
    z = np.where(bad, np.nan, z)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        t = (x - z).astype(np.float32).astype(np.float64)
        c = np.where(s > 0, np.minimum(np.rint(t / np.where(s > 0, s, 1.0)), 15.0), 0.0)
    return z, s, c


def held(x, round_to, least_step):
    """z + s c, unrounded."""
    z, s, c = hold(x, round_to, least_step)
    return z + s * c


def scales(q, keys, values, p, scale):
    """What rounding errors of one row's attention scale with, for its visible keys
    (z, s, c each) [n, D] or [n, 1] and weights p [n]: the largest scale * sum |q| (|z| + 31 s)
    of a logit, and the sums of p (|z| + s c) and p (|z| + 16 s) of the values, per element."""
    zk, sk, _ = keys
    zv, sv, cv = values
    logit = scale * np.abs(q).sum() * (np.abs(zk) + 31 * sk).max()
    return logit, p @ (np.abs(zv) + sv * cv), p @ (np.abs(zv) + 16 * sv)
