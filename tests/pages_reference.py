"""Plain 64-bit forms of rotary positions, appending to a paged cache and attention over it, and how far a kernel's result may
be from them.  Written from the definitions with numpy; nothing here comes from the package.
"""
import math

import numpy as np

EPS2 = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}  # half a step, relative to the value


def rotate(x, positions, frequency, axis, halves, dtype, inverse=False):
    """x [tokens, heads, dim] in 64 bits, positions [axes, tokens]: the rotated values and their tolerance.

    Tolerance, for a pair (a, b): the angle as a fraction of a turn is an fp32 number of at most 1/2 (off by 2^-26 of a turn,
    2^-23.3), after products in 64 bits (2^-52 of the angle); sine and cosine are off by a step at most (2^-23 here); the two
    products and their sum by half a step each (2^-24): all times |a| + |b|, together below 2^-21.6; and the type's rounding.
    """
    half = len(frequency)
    y, tol = x.copy(), np.zeros_like(x)
    for i in range(half):
        a, b = (i, i + half) if halves else (2 * i, 2 * i + 1)
        t = positions[axis[i]].astype(np.float64) * frequency[i]
        c, s = np.cos(t)[:, None], np.sin(t)[:, None] * (-1.0 if inverse else 1.0)
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        size = np.abs(x[..., a]) + np.abs(x[..., b])
        off = size * (2.0 ** -21.6 + 2.0 ** -51 * np.abs(t)[:, None])
        for ch in (a, b):
            tol[..., ch] = off + EPS2[dtype] * (np.abs(y[..., ch]) + off)
    return y, tol * 1.001 + 1e-38


def visible(n, rows, window, sinks):
    """[n, rows]: which rows each of the last n tokens sees."""
    p, x = (rows - n + np.arange(n))[:, None], np.arange(rows)
    seen = x <= p
    return seen & ((x > p - window) | (x < sinks)) if window else seen


def attend(q, k, v, seen, scale, dtype, one_bf16):
    """One sequence.  q [n, Hq, d], k, v [rows, H, d] in 64 bits, seen [n, rows].  Returns out, lse and their tolerances.

    Tolerance of an output, with A = sum p |v| and p the exact probabilities:
      - its own rounding: half a step of the type;
      - a probability as the matrix instruction's operand: none for float32; for bfloat16 two of them together (2^-15), or
        one (2^-8) where `one_bf16`;
      - logits: d products summed in fp32, each off by half a step of the running sum: (d + 4) 2^-23 c sum |q k|, an absolute
        error of the exponent, hence a relative one of p, twice (numerator and sum);
      - fp32 sums over n keys: n 2^-24 A, chunks of them joined, and exp2 (2^-21 relative).
    """
    n, hq, d = q.shape
    rows, h = k.shape[0], k.shape[1]
    g = hq // h
    out, lse = np.zeros((n, hq, d)), np.full((n, hq), -np.inf)
    tol, ltol = np.zeros((n, hq, d)), np.zeros((n, hq))
    some = seen.any(1) if rows else np.zeros(n, bool)
    if not some.any():
        return out, lse, tol + 1e-30, ltol
    need = seen.any(0)
    p_err = 0.0 if dtype == "f32" else EPS2["bf16"] if one_bf16 else 2.0 ** -15
    for hh in range(hq):
        kk, vv, qq = np.where(need[:, None], k[:, hh // g], 0.0), np.where(need[:, None], v[:, hh // g], 0.0), q[:, hh]
        x = np.where(seen, scale * (qq @ kk.T), -np.inf)
        top = np.where(some, x.max(1), 0.0)
        p = np.exp(x - top[:, None])
        l = np.where(some, p.sum(1), 1.0)
        p /= l[:, None]
        out[:, hh] = p @ vv
        lse[:, hh] = np.where(some, top + np.log(l), -np.inf)
        a = p @ np.abs(vv)
        size = np.where(seen, np.abs(qq) @ np.abs(kk).T, 0.0).max(1)
        ds = scale * (d + 4) * 2.0 ** -23 * size + np.where(seen, np.abs(x), 0.0).max(1) * 2.0 ** -22
        r = seen.sum(1)
        rel = p_err + 2 * ds + (2 * r + 64) * 2.0 ** -24 + 2.0 ** -20
        tol[:, hh] = EPS2[dtype] * np.abs(out[:, hh]) + rel[:, None] * a
        ltol[:, hh] = np.where(some, ds + (r + 64) * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -23 * np.abs(np.where(some, lse[:, hh], 0.0)), 0.0)
    return out, lse, tol * 1.001 + 1e-30, ltol


def compare(got, want, tol, what):
    """Finite values within tol; the same infinities, and NaN where the definition gives NaN."""
    got = got.detach().double().cpu().numpy()
    assert got.shape == want.shape, what
    assert np.array_equal(np.isnan(want), np.isnan(got)), what + ": NaN in other places"
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), what + ": infinities"
    ok = np.isfinite(want)
    err = np.abs(got[ok] - want[ok])
    over = ~(err <= tol[ok])
    assert not over.any(), "%s: %d of %d beyond the tolerance, worst %.3g (allowed %.3g)" % (
        what, over.sum(), over.size, err[over].max(), tol[ok][over][err[over].argmax()])


def scale_of(dim, scale=0.0):
    return float(np.float32(scale if scale > 0 else 1.0 / math.sqrt(dim)))
