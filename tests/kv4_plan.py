"""What an attention over the 4-bit cache runs on, from the library's host code."""
import collections
import ctypes

import paper_2609_33390_amd as brisk

Plan = collections.namedtuple("Plan", "width rows waves lanes tiles runs run by_length")


def plan4(B, L, H, Hkv, D, prefix, most):
    """``width``, ``rows``, ``waves`` and ``lanes`` name the kernel; None where no kernel reads own keys."""
    fn = getattr(brisk.lib(), "_ZN5brisk23kv4_attention_plan_infoEiiiiiiiPi")    # internal, not part of the C ABI
    fn.restype = ctypes.c_bool
    out = (ctypes.c_int * 8)()
    return Plan(*out) if fn(B, L, H, Hkv, D, prefix or 0, most, out) else None
