"""Plain 64-bit forms of the K/V store operators, and how far a kernel's result may be from them.

Written from the definitions with numpy; nothing here comes from the package.
"""
import numpy as np
import torch

EPS2 = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # half a step, relative to the value


def quantise(x):
    """[tokens, heads, dim] -> e4m3 codes [heads, tokens, dim] and scale bytes [heads, tokens], by exact arithmetic."""
    x = np.asarray(x.detach().double().cpu()).transpose(1, 0, 2)
    finite = np.where(np.isfinite(x), np.abs(x), 0.0)
    big = finite.max(-1)
    e = np.full(big.shape, -15)
    for p in range(-15, 7):
        e = np.where(big > 448.0 * 2.0 ** p, p + 1, e)
    y = x / 2.0 ** e[..., None]
    a = np.minimum(np.where(np.isnan(y), 0.0, np.abs(y)), 448.0)
    _, k = np.frexp(np.maximum(a, 2.0 ** -6))  # a in [2^(k-1), 2^k)
    step = 2.0 ** (k - 4.0)                    # eight steps to a binade; 2^-9 below 2^-6
    n = np.rint(a / step).astype(np.int64)     # 0 .. 16
    k = np.where(n == 16, k + 1, k)
    n = np.where(n == 16, 8, n)
    code = np.where(n < 8, n, ((k - 1 + 7) << 3) + (n - 8))  # subnormals have exponent field 0
    code = np.where(np.isnan(x), 0x7F, code)
    sign = np.signbit(y) & ~np.isnan(x)
    return (code | (sign.astype(np.int64) << 7)).astype(np.uint8), (e + 127).astype(np.uint8)


def values(code, scale):
    """The numbers codes [heads, rows, dim] and scales [heads, rows] stand for, in 64 bits."""
    c = np.asarray(code.cpu() if torch.is_tensor(code) else code).astype(np.int64)
    s = np.asarray(scale.cpu() if torch.is_tensor(scale) else scale).astype(np.int64)
    m, e = c & 7, (c >> 3) & 15
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((c & 0x7F) == 0x7F, np.nan, v)
    return np.where(c & 0x80, -v, v) * 2.0 ** (s - 127.0)[..., None]


def attend(q, k, v, seen, scale, fmt, out_dtype):
    """One sequence.  q [n, Hq, d], k, v [rows, H, d] in 64 bits, seen [n]: how many of the rows each token sees.
    Returns out, lse and their tolerances.

    Tolerance of an output, with A = sum p |v| and p the exact probabilities:
      - its own rounding: half a step of the type;
      - a probability as the matrix instruction's operand: bf16 (2^-8) for bf16 rows, f16 (2^-11, and 2^-25 absolute
        for what is subnormal there, relative to a largest probability that is at least 2^-8 of the reference) for 8-bit
        rows, none for float32 rows;
      - logits: d products of fp32 sums, each off by half a step of the running sum: (d + 4) 2^-23 c sum |q k|, an
        absolute error of the exponent, hence a relative one of p, twice (numerator and sum); the f16 query operand of
        8-bit rows adds 2^-24 max |q| sum |k|;
      - fp32 sums over n keys: n 2^-24 A, n chunks of them joined, and exp2 (2^-21 relative).
    """
    n, hq, d = q.shape
    h = k.shape[1] if k.ndim == 3 else 1
    g = hq // h
    out, lse = np.zeros((n, hq, d)), np.full((n, hq), -np.inf)
    tol, ltol = np.zeros((n, hq, d)), np.zeros((n, hq))
    for t in range(n):
        r = int(max(0, min(seen[t], k.shape[0])))
        if r == 0:
            continue
        for hh in range(hq):
            kk, vv, qq = k[:r, hh // g], v[:r, hh // g], q[t, hh]
            x = scale * (kk @ qq)
            top = x.max()
            if top == -np.inf:
                continue
            p = np.exp(x - top)
            l = p.sum()
            p /= l
            out[t, hh] = p @ vv
            lse[t, hh] = top + np.log(l)
            a, va = p @ np.abs(vv), np.abs(vv).sum(0)
            ds = scale * (d + 4) * 2.0 ** -23 * (np.abs(kk) @ np.abs(qq)).max() + np.abs(x[np.isfinite(x)]).max() * 2.0 ** -22
            if fmt == "kv8":
                ds += scale * 2.0 ** -24 * np.abs(qq).max() * np.abs(kk).sum(1).max()
            p_err = {"f32": 0.0, "bf16": EPS2["bf16"], "kv8": EPS2["f16"]}[fmt]
            tol[t, hh] = EPS2[out_dtype] * np.abs(out[t, hh]) + (p_err + 2 * ds + (2 * r + 64) * 2.0 ** -24 + 2.0 ** -20) * a
            if fmt == "kv8":
                tol[t, hh] += 2.0 ** -25 * va / l
            ltol[t, hh] = ds + (r + 64) * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -23 * abs(lse[t, hh])
    return out, lse, tol * 1.001 + 1e-30, ltol


def compare(got, want, tol, what):
    """Finite values within tol; the same infinities, and NaN where the definition gives NaN."""
    got = got.detach().double().cpu().numpy()
    assert got.shape == want.shape, what
    bad_want = ~np.isfinite(want)
    assert np.array_equal(np.isnan(want), np.isnan(got)), what + ": NaN in other places"
    inf = bad_want & ~np.isnan(want)
    assert np.array_equal(got[inf], want[inf]), what + ": infinities"
    ok = ~bad_want
    err = np.abs(got[ok] - want[ok])
    over = err > tol[ok]
    assert not over.any(), "%s: %d of %d beyond the tolerance, worst %.3g (allowed %.3g)" % (
        what, over.sum(), over.size, err[over].max(), tol[ok][over][err[over].argmax()])
