"""Checks of the decoding operators that hold for long reductions too, where the bound of the worst case is larger than the
result: blocks of a row against the 64-bit values, by their L2 norms."""
from __future__ import annotations

import numpy as np

import few_reference as ref

COLS = 64  # of a block
# Relative to a block's norm.  bf16: `a` and the output are rounded once each, by at most 2^-8 of an element; a block's norm
# of both is at most about sqrt(2) 2^-8 = 5.5e-3 where the roundings of `a` are as good as independent, and twice that is allowed.  fp32:
# sums of up to 8192 terms, off by sqrt(8192) 2^-24 = 5e-6 of their size as rounding goes, some 2e-5 after two of them.
LIMIT = {"bf16": 1.1e-2, "f32": 1e-4}


def held(packed, scales, fmt, group):
    """What an fp32 sum holds of a weight: its magnitude, or (INT4) its code and 8 apart, in scales."""
    if fmt == ref.FP4:
        return np.abs(ref.values(packed, scales, fmt, group))
    s = np.repeat(np.abs(ref.f64(scales)), group, axis=-1)[..., :2 * packed.shape[-1]]
    return (ref.codes_of(packed) + 8.0) * s


def off(got, want):
    """[rows, blocks] of what blocks are off by, relative to their norm."""
    rows, n = want.shape
    out = np.empty((rows, -(-n // COLS)))
    for b in range(out.shape[1]):
        lo = min(b * COLS, max(n - COLS, 0))  # (the last block is as long as the others)
        w = want[:, lo:lo + COLS]
        out[:, b] = np.linalg.norm(got[:, lo:lo + COLS] - w, axis=1) / np.linalg.norm(w, axis=1)
    return out


def check(got, want, dtype, what):
    d = off(ref.f64(got), want)
    assert np.isfinite(d).all(), what
    at = np.unravel_index(np.argmax(d), d.shape)
    assert d[at] < LIMIT[dtype], (what, at, d[at])
