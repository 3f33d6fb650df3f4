"""The operators over a paged cache of several sequences in 64 bits, from their definition (tests only)."""
import math

import torch

F8 = torch.float8_e4m3fn


def place(kind, h, key, dim):
    """Byte offsets of K[key, dim] and V[key, dim] in a chunk, element by element from the layout's text."""
    ke, size = {"f32": (4, 4), "bf16": (8, 2), "fp8": (16, 1)}[kind]
    d = min(ke, h // 4)
    for kt in range(4):
        for r in range(16):
            at = 16 * kt + r if kind == "f32" else 32 * (kt // 2) + 8 * (r // 4) + 4 * (kt % 2) + r % 4 if kind == "bf16" else 16 * (r // 4) + 4 * kt + r % 4
            if at == key:
                hp, g = dim // (4 * d), dim % (4 * d) // d
                k = ((kt * (h // (4 * d)) + hp) * 64 + 16 * g + r) * d + dim % d
    ks, g = key // (4 * ke), key % (4 * ke) // ke
    v = 64 * h + ((dim // 16 * (16 // ke) + ks) * 64 + 16 * g + dim % 16) * ke + key % ke
    return k * size, v * size


def exponent(x):
    """Exponents of the scales of x [..., dim] (64 bits): the least e with max|x| 2^-e <= 448."""
    top = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448))
    e = torch.where(torch.ldexp(top, -e) > 448, e + 1, torch.where(torch.ldexp(top, 1 - e) <= 448, e - 1, e))
    return torch.where(top == 0, 0.0, e).clamp(-100, 120)


def held(x):
    """(values that an 8-bit cache holds of x, how far x may be moved without changing them, their spacing)."""
    unit = torch.exp2(exponent(x))
    y = torch.where(x.isfinite(), x / unit, 0.0)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    z = torch.round(y / step) * step
    border = (0.5 - (y / step - torch.round(y / step)).abs()) * step * unit
    return torch.where(x.isfinite(), z * unit, math.nan), border, step * unit


def prepared(x, gain, eps, angles, rot, inter):
    """x [rows, heads, dim] normalised and rotated; angles [rows, rot/2, 2] (cos, sin)."""
    x = x.double()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()
    if not rot:
        return x
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :rot // 2], x[..., rot // 2:rot])
    c, s = angles.double()[:, None, :, 0], angles.double()[:, None, :, 1]
    a, b = a * c - b * s, b * c + a * s
    y = torch.stack([a, b], -1).flatten(-2) if inter else torch.cat([a, b], -1)
    return torch.cat([y, x[..., rot:]], -1)


def attention(q, k, v, first, scale):
    """Rows q [n, heads, dim] at positions first .. over k, v [tokens, kv heads, dim]: (out, sum of p|v|, largest sum of |q||k| times scale)."""
    n, heads, h = q.shape
    group = heads // k.shape[1]
    q, k, v = q.double(), k.double().repeat_interleave(group, 1), v.double().repeat_interleave(group, 1)
    pos = torch.arange(first, first + n, device=q.device)
    hidden = torch.arange(k.shape[0], device=q.device)[None, :] > pos[:, None]
    s = torch.einsum("nhd,khd->hnk", q, torch.nan_to_num(k, 0.0, 0.0, 0.0) if bool(hidden.any()) and not bool(k.isfinite().all()) else k) * scale
    s = s.masked_fill(hidden, -math.inf)
    p = torch.where(hidden, 0.0, torch.softmax(s, -1)) if k.shape[0] else s
    p = torch.nan_to_num(p, 0.0) if k.shape[0] and bool((pos < 0).any()) else p
    big = torch.where(hidden, 0.0, torch.einsum("nhd,khd->hnk", q.abs(), torch.nan_to_num(k.abs(), 0.0, 0.0, 0.0))).amax(-1).t() * scale if k.shape[0] else torch.zeros(n, heads, device=q.device)
    clean = torch.nan_to_num(v, 0.0, 0.0, 0.0)
    out = torch.einsum("hnk,khd->nhd", p, clean)
    seen = (~hidden).double()
    for bad, value in ((v.isnan(), math.nan), (v == math.inf, math.inf), (v == -math.inf, -math.inf)):
        if bool(bad.any()):
            out = torch.where(torch.einsum("nk,khd->nhd", seen, bad.double()) > 0, out + value, out)
    return out, torch.einsum("hnk,khd->nhd", p, clean.abs()), big
