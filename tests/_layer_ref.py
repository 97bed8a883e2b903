"""The operators around a layer's cache from their definitions, in 64 bits: what the CUDA calls are compared with.

Tolerances (each rounding counts torch.finfo(t).eps / 2: bf16 2^-8, fp16 2^-11, fp32 2^-24, e4m3 2^-4 of the value):
  attention   A logit is a sum of 128 exact products, each cut to 2^-23 of the magnitudes: 2^-16 sm_scale sum |q k|; its scaling, the
              reference's subtraction and the exponential's argument add 2^-22 (|x| + max |x| + 16). Of that, eps_x, a weight is off by
              2 eps_x relative (e^eps - 1 < 2 eps), and by its rounding: bf16 2^-8, or 2^-16 in two parts; f16 2^-11, and 2^-25 of
              the largest p 2^ev where it is subnormal (the largest weight of a sum is at least 1, of the smallest code's step 2^-9
              upwards). n rows make n / 16 fp32 steps of a sum and as many joins: 2^-22 (n / 16 + 64) of the sum of magnitudes.
              Outputs: 2^-8 |o| + (rounding + 2 eps_x + steps) sum p |v| (8 bits: + 2^-25 max(p 2^ev) sum |code|) / sum p;
              log-sum-exp: eps_x + steps + 2^-22 |lse|.
  add_norm    the sum: 2^-8 |s|. y: rsqrt 2^-22, the sum of squares dim fp32 additions of a tree at most 32 deep per thread plus a
              butterfly, halved by the root: 2^-19 together with its products; then 2^-8 in bf16, or half an e4m3 step.
  axes        one bf16 rounding, 2^-8 |z|, plus 2^-19 (|y_a| + |y_b|) for the fp32 chain before it, as for one axis.
"""
from __future__ import annotations

import math

import torch

E4M3_MAX = 448.0


def e4m3_table(dev):
    v = []
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        mag = math.nan if c & 127 == 127 else (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
        v.append(-mag if c & 128 else mag)
    return torch.tensor(v, dtype=torch.float64, device=dev)


def dense(q, k_of, v_of, lens, T, group, sm_scale, causal, window, weight_eps):
    """q [B, T, Hq, 128]; k_of(b), v_of(b): ([n, Hkv, 128] values, [n] which rows exist[, [n, Hkv] 2^ev]) in 64 bits. Outputs, log-sum-exps
    and what either may be off by."""
    B, _, hq, _ = q.shape
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.full(q.shape[:3], -math.inf, dtype=torch.float64, device=q.device)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(B):
        n = int(lens[b])
        if n <= 0:
            continue
        (k, ok), (v, ev) = k_of(b), v_of(b)
        heads = torch.arange(hq, device=q.device) // group
        for t in range(T):
            here = n - T + t
            pos = torch.arange(n, device=q.device)
            see = ok & (pos < (here + 1 if causal else n))
            if window:
                see = see & (pos > here - window)
            if not bool(see.any()):
                continue
            kk, vv = k[see][:, heads], v[see][:, heads]  # [s, Hq, 128]
            qq = q[b, t].double()
            x = (kk * qq).sum(-1).T * sm_scale  # [Hq, s]
            size = torch.where(x == -math.inf, 0.0, x.abs())  # (a logit of -inf has weight 0 exactly)
            eps = 2.0 ** -16 * (kk.abs() * qq.abs()).sum(-1).T * sm_scale + 2.0 ** -22 * (size + size.amax(-1, keepdim=True) + 16)
            eps = torch.where(x == -math.inf, 0.0, eps)
            p = torch.softmax(x, -1)
            out[b, t] = torch.einsum("hs,shd->hd", p, vv)
            lse[b, t] = torch.logsumexp(x, -1)
            steps = 2.0 ** -22 * (n / 16 + 64)
            mag = torch.einsum("hs,shd->hd", p * (weight_eps + 2 * eps + steps), vv.abs())
            if ev is not None:
                e = ev[see][:, heads].T  # [Hq, s]
                mag = mag + 2.0 ** -25 * (p * e).amax(-1)[:, None] * (vv.abs() / ev[see][:, heads][..., None]).sum(0)
            tol[b, t] = 2.0 ** -8 * out[b, t].abs() + mag
            ltol[b, t] = (p * eps).sum(-1) + steps + 2.0 ** -22 * lse[b, t].abs()
    return out, lse, tol, ltol


def check_close(got, want, tol, what):
    """Equal within tol, and not finite in the same places with the same values."""
    got = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), f"{what}: other infinities"
    off = (got - want).abs()[fine] - tol[fine]
    assert off.numel() == 0 or float(off.max()) <= 0, f"{what}: off by {float((got - want).abs()[fine].max())}, {float(off.max())} over the tolerance"


def exponents(y):
    """The smallest e in -100 .. 120 with max |y| <= 448 2^e over the last axis' finite elements."""
    a = torch.where(torch.isfinite(y), y.abs(), torch.zeros_like(y)).amax(-1)
    e = torch.ceil(torch.log2(a / E4M3_MAX)).clamp(-100, 120)
    e = torch.where(a > E4M3_MAX * torch.exp2(e), e + 1, e)
    return torch.where(a <= E4M3_MAX * torch.exp2(e - 1), e - 1, e).clamp(-100, 120)
