"""The 8-bit cache operators from their definitions, in 64 bits with numpy: what the CUDA calls are compared with.

Tolerances (each rounding counts torch.finfo(t).eps / 2: bf16 2^-8, fp16 2^-11, fp32 2^-24, e4m3 2^-4 of the value):
  norm_rope   one bf16 rounding, 2^-8 |z|, plus the fp32 chain before it: the sum of squares (tree, < 2^-21), rsqrt (2^-22),
              two products, an angle rounded to 2^-25 of a turn (2 pi 2^-25 < 2^-22) and its sine (2^-22), the turn: together
              below 2^-19 (|y_a| + |y_b|).
  append      codes are the nearest ones, ties to even: equal bit for bit where the rows are taken as they are (a product with
              a power of two is exact); behind a norm the value may also lie 2^-19 (|y_a| + |y_b|) beyond half a step.
  scores      products are exact, at most 128 fp32 sums, each cut to 2^-23 of the magnitudes: 2^-16 sum |q_j k_j|; and 2^-149, the
              distance of neighbouring fp32 values below 2^-126: a score of smaller magnitude than that has no fp32 form but 0.
  attention   logits as the scores plus three fp32 roundings of numbers up to |x| + 128 in the log2 domain:
              eps = 2^-16 sm_scale sum |q k| + 2^-21 (|x| + 128). A weight is off by that and by one f16 rounding, 2^-11 of it, or
              2^-25 where it is subnormal; the largest weight of a sum is at least 1, so that is 2^-25 of the largest p 2^ev, times
              the code. Outputs: 2^-8 |o| + (2^-11 + 2^-15 + 2 eps) sum p |v| + 2^-25 max(p 2^ev) sum |code|, the log-sum-exp:
              eps + 2^-21 (|lse| + 1) (its sum is of unrounded weights).
"""
from __future__ import annotations

import numpy as np

E4M3 = np.array([np.nan if c & 127 == 127 else (-1.0 if c & 128 else 1.0) * (
    (c & 7) * 2.0 ** -9 if (c >> 3) & 15 == 0 else (8 + (c & 7)) * 2.0 ** (((c >> 3) & 15) - 10)) for c in range(256)])
_MAG = E4M3[:127]                          # 0 .. 448
_MID = (_MAG[:-1] + _MAG[1:]) / 2
EXP_MIN, EXP_MAX = -100, 120


def encode(x):
    """Nearest e4m3 codes of float64 values, ties to the even code, saturating; a NaN gives 0x7f."""
    a = np.abs(x)
    i = np.searchsorted(_MID, a, side="left")
    i = np.where((i < 126) & (a == _MID[np.minimum(i, 125)]) & (i % 2 == 1), i + 1, i)
    code = np.where(np.signbit(x), i + 128, i)
    return np.where(np.isnan(x), 127, code).astype(np.uint8)


def half_step(x, e):
    """Half the distance of neighbouring values around x in a block of exponent e."""
    a = np.maximum(np.abs(x) * 2.0 ** -e, 2.0 ** -6)
    return np.ldexp(1.0, (np.floor(np.log2(a)) - 4).astype(int)) * 2.0 ** e


def norm_rope(x, pos, weight, norm, eps, inv_freq, interleaved, rot_scale=1.0):
    """x [tokens, heads, D] float64. Returns (z, |y_a| + |y_b| of each element's pair)."""
    y = x
    if norm:
        y = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
        if weight is not None:
            y = y * weight
    z, mag = y.copy(), np.abs(y) * 2
    if inv_freq is not None:
        half = len(inv_freq)
        ang = pos.astype(np.float64)[:, None] * inv_freq.astype(np.float64)
        c, s = np.cos(ang)[:, None] * rot_scale, np.sin(ang)[:, None] * rot_scale
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        z[..., a] = y[..., a] * c - y[..., b] * s
        z[..., b] = y[..., b] * c + y[..., a] * s
        mag[..., a] = mag[..., b] = (np.abs(y[..., a]) + np.abs(y[..., b])) * max(1.0, abs(rot_scale))
    return z, mag


def need_exponent(amax):
    e = EXP_MIN
    if amax > 0:
        m, ex = np.frexp(amax)  # amax = m 2^ex
        e = int(ex) - 9 + (1 if m > 0.875 else 0)
    return min(max(e, EXP_MIN), EXP_MAX)


def append(codes, scale, rows_of, n, new, block):
    """New rows [T, H, D] float64 of one sequence of n tokens into codes [rows, H, D] and scale [H, blocks] (numpy, in place).
    rows_of: position -> cache row. Returns {(block row, head): exponent} of the blocks written."""
    T = new.shape[0]
    first = n - T
    done = {}
    for begin in range(first // block * block, n, block):
        lo, hi = max(first, begin), min(n, begin + block)
        home = rows_of(begin)
        assert home % block == 0
        for h in range(new.shape[1]):
            part = new[lo - first:hi - first, h]
            fin = np.abs(part[np.isfinite(part)])
            e = need_exponent(fin.max() if fin.size else 0.0)
            if lo > begin:
                old = min(max(int(scale[h, home // block]), 27), 247) - 127
                e = max(e, old)
                if e > old:
                    for s in range(begin, lo):
                        codes[rows_of(s), h] = encode(E4M3[codes[rows_of(s), h]] * 2.0 ** (old - e))
            for s in range(lo, hi):
                with np.errstate(invalid="ignore"):
                    codes[rows_of(s), h] = encode(new[s - first, h] * 2.0 ** -e)
            scale[h, home // block] = e + 127
            done[(home, h)] = e
    return done


def values(codes, scale, block):
    """float64 values of codes [rows, H, D] with scale bytes [H, blocks]."""
    f = 2.0 ** (np.clip(scale.astype(np.float64), 27, 247) - 127)
    rows = np.arange(codes.shape[0])
    return E4M3[codes] * f[:, rows // block].T[..., None]


def scores(q, keys):
    """q [T, d], keys [n, d] float64: (scores [T, n], sum of magnitudes)."""
    return q @ keys.T, np.abs(q) @ np.abs(keys).T


def attention(q, k, v, f, sm_scale):
    """q [H, D], k, v [c, G, D] of the selected rows, f [c, G] the scales of v's rows: (out [H, D], lse [H], tolerance of out,
    tolerance of lse)."""
    H, G = q.shape[0], k.shape[1]
    if k.shape[0] == 0:
        return np.zeros_like(q), np.full(H, -np.inf), np.zeros_like(q), np.zeros(H)
    k, v, f = np.repeat(k, H // G, 1), np.repeat(v, H // G, 1), np.repeat(f, H // G, 1)
    x = np.einsum("hd,chd->hc", q, k) * sm_scale
    mag = 2.0 ** -16 * np.einsum("hd,chd->hc", np.abs(q), np.abs(k)) * sm_scale
    top = x.max(-1, keepdims=True)
    w = np.exp(x - top)
    tot = w.sum(-1, keepdims=True)
    p = w / tot
    lse = (top + np.log(tot))[:, 0]
    out = np.einsum("hc,chd->hd", p, v)
    eps = (mag + 2.0 ** -21 * (np.abs(x) + 128)).max(-1)
    tol = 2.0 ** -8 * np.abs(out) + (2.0 ** -11 + 2.0 ** -15 + 2 * eps)[:, None] * np.einsum("hc,chd->hd", p, np.abs(v))
    tol += 2.0 ** -25 * (p * f.T).max(-1)[:, None] * (np.abs(v) / f[..., None]).sum(0)
    return out, lse, tol, eps + 2.0 ** -21 * (np.abs(lse) + 1)
