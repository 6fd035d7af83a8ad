"""The decoding operators in 64 bits (numpy), with bounds on how far the kernels may be off: every rounding by half a
unit of the type it goes to, every fp32 sum by its length times 2^-24 of the sum of its terms' magnitudes."""
from __future__ import annotations

import numpy as np

import moe_inputs as mi

FP4_GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
FP4, INT4 = 0, 1
EPS32 = 2.0 ** -24  # half a unit in the last place, relative
HALF = {"bf16": 2.0 ** -8, "f32": EPS32}


def f64(a):
    return mi.bf16_bits_to_f32(a).astype(np.float64) if a.dtype == np.uint16 else a.astype(np.float64)


def codes_of(packed):
    """[..., cols] codes of [..., cols / 2] bytes: the even column in the low half."""
    out = np.empty((*packed.shape[:-1], 2 * packed.shape[-1]), np.int64)
    out[..., 0::2] = packed & 15
    out[..., 1::2] = packed >> 4
    return out


def pack(codes):
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def values(packed, scales, fmt, group):
    """64-bit values of codes [..., cols / 2] under scales (bytes, or bf16 bits)."""
    c = codes_of(packed)
    cols = c.shape[-1]
    if fmt == FP4:
        v = np.where(c >= 8, -1.0, 1.0) * FP4_GRID[c & 7]
        s = 2.0 ** (scales.astype(np.float64) - 127.0)
    else:
        v = c - 8.0
        s = f64(scales)
    return v * np.repeat(s, group, axis=-1)[..., :cols]


def most(packed, scales, fmt, group):
    """What an fp32 sum over a weight may hold of it: its magnitude, or (INT4) up to 144 units of its scale."""
    if fmt == FP4:
        return np.abs(values(packed, scales, fmt, group))
    return np.repeat(np.abs(f64(scales)), group, axis=-1)[..., :2 * packed.shape[-1]] * 144.0


def quantize(w, fmt, group):
    """(codes, scales) of w [rows, cols] float64 holding fp32 or bf16 numbers; scales as bytes or bf16 bits."""
    rows, cols = w.shape
    n = -(-cols // group)
    full = np.zeros((rows, n * group))
    full[:, :cols] = w
    full = full.reshape(rows, n, group)
    m = np.abs(full).max(axis=2)
    if fmt == FP4:
        e = np.frexp(np.where(m > 0, m, 1.0))[1] - 1  # floor(log2)
        s = np.where(m > 0, np.maximum(e - 2 + 127, 1), 1)
        q = np.abs(full) / 2.0 ** (s - 127.0)[..., None]
        edge = (FP4_GRID[1:] + FP4_GRID[:-1]) / 2
        up = np.array([False, True, False, True, False, True, False])  # a tie goes to the even code
        code = ((q[..., None] > edge) | ((q[..., None] == edge) & up)).sum(axis=-1)
        code = np.where(np.signbit(full), code + 8, code)
        return pack(code.reshape(rows, n * group)[:, :cols]), s.astype(np.uint8)
    f, e = np.frexp(m / 7.0)
    s = np.ldexp(np.rint(f * 256.0), e - 8)
    q = np.divide(full, s[..., None], out=np.zeros_like(full), where=s[..., None] > 0)
    code = np.clip(np.rint(q), -8, 7).astype(np.int64) + 8
    return pack(code.reshape(rows, n * group)[:, :cols]), mi.f32_to_bf16_bits(s.astype(np.float32))


def product(x, W, W_most, x_err=0.0):
    """x W^T [rows, n] and a bound on what fp32 sums of it may be off by; x_err: how far x itself may be off."""
    y = x @ W.T
    sums = np.abs(x) @ W_most.T
    err = (W.shape[1] + 40) * EPS32 * sums
    if np.any(x_err):
        err = err + x_err @ np.abs(W).T
    return y, err


def layer(x, idx, w, gate, up, down, dtype):
    """out [N,H] and its bound.  gate, up, down: functions e -> (values, magnitudes) of an expert's matrix."""
    N, H = x.shape
    out, err = np.zeros((N, H)), np.zeros((N, H))
    half = HALF[dtype]
    for e in np.unique(idx):
        n, k = np.nonzero(idx == e)
        g, dg = product(x[n], *gate(e))
        u, du = product(x[n], *up(e))
        s = 1.0 / (1.0 + np.exp(-g))
        a = g * s * u
        # silu' is within [-0.1, 1.1]; the function itself in fp32: a few units of its last place
        da = 1.1 * dg * np.abs(u) + np.abs(g * s) * du + 1.1 * dg * du + 8 * EPS32 * np.abs(a)
        da = da + half * (np.abs(a) + da) + (1e-37 if dtype == "bf16" else 1e-44)
        y, dy = product(a, *down(e), da)
        wk = w[n, k][:, None]
        out[n] += wk * y
        err[n] += np.abs(wk) * dy + (2e-6 + 64 * EPS32) * np.abs(wk * y)
    return out, err + half * (np.abs(out) + err)


def check(got, want, bound, what):
    got = f64(got)
    assert np.isfinite(got).all(), what
    over = np.abs(got - want) - bound
    at = np.unravel_index(np.argmax(over), over.shape)
    assert over[at] <= 0, (what, at, got[at], want[at], bound[at])
