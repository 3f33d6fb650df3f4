"""Attention over chosen keys in 64 bits, from its definition, and the tolerances of the operators that are compared with it (tests only).

Tolerances, fixed before the first run.  Rounding to a type is off by at most half a step (bf16 2^-8, fp32 2^-24 of the value).  A score is a sum of h products,
off by E = h 2^-24 scale sum|q||k| at most; weights are off by 2E from the scores of both sides of the softmax and 2^-20 from the exponentials (an argument of
up to 2^3 that counts, in steps of 2^-24, and an ulp of the function), bf16 rows round each by 2^-8 more; sums over n keys add n 2^-24; all of it times
sum p|v|; then one rounding.
"""
import math

import torch

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def in_window(pos, keys, window, sinks):
    """[rows, keys]: what rows at these positions see of the keys 0 .. keys - 1."""
    j = torch.arange(keys, device=pos.device)[None, :]
    return (j <= pos[:, None]) & ((j > pos[:, None] - window) | (j < sinks))


def attention(q, k, v, seen, scale):
    """q [n, heads, dim] over k, v [keys, kv heads, dim], seen [n, keys]: (out, sum of p|v|, largest sum of |q||k| times scale)."""
    group = q.shape[1] // k.shape[1]
    q, k, v = q.double(), k.double().repeat_interleave(group, 1), v.double().repeat_interleave(group, 1)
    hidden = ~seen
    usual = torch.nan_to_num(k, 0.0, 0.0, 0.0)
    s = torch.einsum("nhd,khd->hnk", q, usual) * scale
    odd = (~k.isfinite()).any(-1).t()[:, None, :]                                   # a K that is not finite: its score is NaN where it is seen
    s = torch.where(odd, math.nan, s).masked_fill(hidden, -math.inf)
    p = torch.where(hidden, 0.0, torch.softmax(s, -1))
    p = torch.where(hidden.all(-1)[:, None], 0.0, p)
    big = torch.where(hidden, 0.0, torch.einsum("nhd,khd->hnk", q.abs(), usual.abs())).amax(-1).t() * scale
    clean = torch.nan_to_num(v, 0.0, 0.0, 0.0)
    out = torch.einsum("hnk,khd->nhd", p, clean)
    for bad, value in ((v.isnan(), math.nan), (v == math.inf, math.inf), (v == -math.inf, -math.inf)):
        if bool(bad.any()):
            out = torch.where(torch.einsum("nk,khd->nhd", seen.double(), bad.double()) > 0, out + value, out)
    return out, torch.einsum("hnk,khd->nhd", p, clean.abs()), big


def close(got, want, tol, what):
    got = got.double()
    assert torch.equal(got.isnan(), want.isnan()), what
    ok = want.isfinite()
    assert torch.equal(got[~ok & ~want.isnan()], want[~ok & ~want.isnan()]), what
    d = torch.where(ok, (got - want).abs() - tol, torch.zeros_like(tol))
    assert float(d.max()) <= 0, f"{what}: {float(d.max())} over the tolerance, difference {float((got - want)[ok].abs().max())}"


def check(dtype, q, out, k, v, seen, scale, what):
    """One sequence's rows; blocks of rows, so that many rows of many keys fit."""
    step = max(1, 2 ** 25 // (q.shape[1] * max(1, k.shape[0])))
    for i in range(0, q.shape[0], step):
        rows = slice(i, i + step)
        want, size, big = attention(q[rows], k, v, seen[rows], scale)
        e = 2 * q.shape[2] * 2.0 ** -24 * big[..., None] + 2.0 ** -20 + k.shape[0] * 2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0.0)
        close(out[rows], want, size * e + (want.abs().nan_to_num(0, 0, 0) + size * e) * HALF[dtype], what)
