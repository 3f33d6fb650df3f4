"""Cases of the operators over a paged cache of several sequences (`KVCache` in the Python binding).

  append   norms of queries and keys per head, rotary positions, K and V into the cache's pages (8 bits: e4m3 codes with one
           power-of-two scale per token and KV head), then the written rows read back, as a program does that hands a
           sequence on: the rotated queries and the cache's values come out.
  attend   causal attention of every sequence's new tokens over its pages: one token each (decoding), a few
           (verification of drafts), a chunk behind a long context, whole prompts.
  read     rows of the cache as values: what a program does that moves a sequence to another place.

Sequences share one pool of pages through a page table (pages in random order); rows of all sequences are packed one behind
the other.  Head counts and widths are those of the shapes in `asd_inputs.SHAPES` (tiny, 7b, 13b, 70b).
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEVICE = "cuda:0" if torch.cuda.is_available() else "cpu"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _case(name, op, dtype, kv, heads, kv_heads, dim, page, seqs, new, ctx, mix, norm=False, rot=0, inter=False, factor=1.0):
    """new: most new rows of a sequence; ctx: most tokens of a sequence with the new ones (0: the new ones are all there is);
    mix: 0 for sequences of one length, else the seed of their lengths."""
    return {"name": name, "op": op, "dtype": dtype, "kv": kv, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page,
            "seqs": seqs, "new": new, "ctx": ctx, "mix": mix, "norm": norm, "rot": rot, "inter": inter, "factor": factor}


def listed():
    return [
        # one decoding step of 48 conversations on the 70B heads: a token each, positions scaled for twice the trained length
        _case("append-decode", "append", "bf16", "fp8", 64, 8, 128, 64, 48, 1, 8192, 3, norm=True, rot=128, factor=2.0),
        # prompts of four requests on the 7B heads, up to 2048 tokens each
        _case("append-prompt", "append", "bf16", "fp8", 32, 32, 128, 64, 4, 2048, 0, 5, rot=128),
        # a fp32 model with a rotation of half of each head in pairs of neighbours: a handful of ragged sequences
        _case("append-f32-part", "append", "f32", "f32", 8, 2, 64, 64, 9, 70, 300, 7, norm=True, rot=32, inter=True),
        # the smallest call: one token of the small fp32 model behind 45 tokens
        _case("attend-one", "attend", "f32", "f32", 4, 4, 64, 64, 1, 1, 45, 0),
        # decoding of 48 conversations of 500 to 8192 tokens on the 70B heads
        _case("attend-decode", "attend", "bf16", "fp8", 64, 8, 128, 64, 48, 1, 8192, 3),
        # one long conversation alone on the 7B heads, cache in bf16
        _case("attend-alone", "attend", "bf16", "bf16", 32, 32, 128, 256, 1, 1, 8192, 0),
        # verification of four drafts and the token before them for eight sequences of the 13B heads
        _case("attend-verify", "attend", "bf16", "fp8", 40, 40, 128, 64, 8, 5, 1031, 11),
        # a chunk of 512 new tokens behind a long document, two requests, 70B heads
        _case("attend-chunk", "attend", "bf16", "fp8", 64, 8, 128, 64, 2, 512, 8707, 13),
        # whole prompts of four requests on the 7B heads, cache in bf16
        _case("attend-prompt", "attend", "bf16", "bf16", 32, 32, 128, 64, 4, 2048, 0, 5),
        # a small fp32 model: ragged chunks of three sequences, grouped heads
        _case("attend-f32", "attend", "f32", "f32", 8, 2, 64, 64, 3, 61, 300, 17),
        # sixteen whole sequences out of an 8-bit cache, 70B heads
        _case("read-whole", "read", "bf16", "fp8", 64, 8, 128, 64, 16, 4096, 0, 19),
        # the last tokens of three sequences of the small fp32 model
        _case("read-last", "read", "f32", "f32", 4, 4, 64, 64, 3, 5, 45, 23),
    ]


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / 1e15 * (8 if c["dtype"] == "f32" else 1))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["append", "attend", "attend", "read"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        # (32-bit rows written in 8 bits come back in 32: a value on a rounding border may then be a whole step off, so they are left out)
        kv = rng.choice([dtype, "fp8", "fp8"]) if op != "append" or dtype == "bf16" else dtype
        dim = rng.choice([64, 128, 128])
        kv_heads, group = rng.choice([(1, 8), (2, 4), (4, 1), (5, 3), (8, 8), (8, 4), (32, 1), (40, 1)])
        wide = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))     # noqa: E731
        new = rng.choice([1, 1, wide(2, 16), wide(16, 2048)])
        ctx = rng.choice([0, new + wide(1, 8192)]) if new > 1 or op == "append" else new + wide(1, 8192)
        rot = rng.choice([dim, dim, dim // 2]) if op == "append" else 0
        c = _case("", op, dtype, kv, kv_heads * group, kv_heads, dim, rng.choice([64, 64, 128, 256]), wide(1, 64), new, ctx,
                  rng.randrange(0, 1000), norm=op == "append" and rng.random() < 0.5, rot=rot, inter=op == "append" and rng.random() < 0.4,
                  factor=rng.choice([1.0, 1.0, 4.0]) if op == "append" else 1.0)
        # the most that the plain form of a batch takes: scores of all sequences padded to the longest, in 32 bits
        if _cost(c) <= most and c["seqs"] * c["heads"] * c["new"] * max(c["ctx"], c["new"]) < 2 ** 31 and c["seqs"] * max(c["ctx"], c["new"]) * c["kv_heads"] * dim < 2 ** 30:
            del c["name"]
            return c


def lens(c):
    """(new rows, tokens) of every sequence; the first is the longest."""
    r, out = random.Random(c["mix"]), []
    for s in range(c["seqs"]):
        new = c["new"] if not c["mix"] or s == 0 else r.randint((c["new"] + 3) // 4, c["new"])
        total = new if not c["ctx"] else c["ctx"] if not c["mix"] or s == 0 else r.randint(max(new, c["ctx"] // 16), c["ctx"])
        out.append((new, total))
    return out


def _token_bytes(c):
    """What a token and KV head take in the cache."""
    return 2 * c["dim"] * {"f32": 4, "bf16": 2, "fp8": 1}[c["kv"]] + (2 if c["kv"] == "fp8" else 0)


def work(c):
    n, e = lens(c), 4 if c["dtype"] == "f32" else 2
    rows, tokens, h = sum(a for a, _ in n), sum(b for _, b in n), c["dim"]
    kv_rows, kv_cache = rows * c["kv_heads"] * 2 * h * e, rows * c["kv_heads"] * _token_bytes(c)
    if c["op"] == "append":
        each = (c["heads"] + c["kv_heads"]) * (4 * h * bool(c["norm"]) + 3 * c["rot"]) + c["kv_heads"] * 4 * h * (c["kv"] == "fp8")
        return {"bytes": rows * c["heads"] * 2 * h * e + 2 * kv_rows + 2 * kv_cache + rows * c["rot"] * 4, "flops": rows * each}
    if c["op"] == "read":
        return {"bytes": kv_cache + kv_rows, "flops": rows * c["kv_heads"] * 2 * h}
    seen = sum(a * b - a * (a - 1) // 2 for a, b in n)      # keys seen by the rows
    return {"bytes": rows * c["heads"] * 2 * h * e + tokens * c["kv_heads"] * _token_bytes(c), "flops": 4 * h * c["heads"] * seen}


def _places(kv, h):
    """(key, dim) of every element of a chunk's K part and of its V part: a cache page holds, per KV head, chunks of 64 tokens, each
    the K values in pieces of 16 bytes as a wave of 64 lanes loads them, then V transposed, likewise (8 bits: then a byte per
    token with the exponent of K's scale + 127, and another 64 for V)."""
    ke = {"f32": 4, "bf16": 8, "fp8": 16}[kv]
    kk = min(ke, h // 4)
    kt, hs, g, r, b = torch.meshgrid(*(torch.arange(n) for n in (4, h // (4 * kk), 4, 16, kk)), indexing="ij")
    key = 16 * kt + r if kv == "f32" else 32 * (kt // 2) + 8 * (r // 4) + 4 * (kt % 2) + r % 4 if kv == "bf16" else 16 * (r // 4) + 4 * kt + r % 4
    k_place = key * h + hs * 4 * kk + g * kk + b
    ht, ks, g, r, b = torch.meshgrid(*(torch.arange(n) for n in (h // 16, 16 // ke, 4, 16, ke)), indexing="ij")
    v_place = (ks * 4 * ke + g * ke + b) * h + 16 * ht + r
    return k_place.reshape(-1), v_place.reshape(-1)


def _quantise(x):
    """x [..., dim] in 32 bits: e4m3 codes and the exponent of the scale."""
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True))
    e = torch.where(m == 0, 0, torch.where(m <= 0.875, e - 9, e - 8)).clamp(-100, 120)
    return torch.ldexp(x, -e).to(torch.float8_e4m3fn), e


def _table(c, n_pos):
    """cos and sin of the positions' angles, positions scaled down by the factor (angles in 64 bits)."""
    j = torch.arange(c["rot"] // 2, dtype=torch.float64, device=DEVICE)
    a = torch.arange(n_pos, dtype=torch.float64, device=DEVICE)[:, None] / c["factor"] * 10000.0 ** (-2 * j / c["rot"])
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def prepare(c, seed):
    gen = torch.Generator(DEVICE).manual_seed(seed)
    n, h, kvh, t = lens(c), c["dim"], c["kv_heads"], TYPES[c["dtype"]]
    rows, longest, page = sum(a for a, _ in n), max(b for _, b in n), c["page"]
    each = (longest + page - 1) // page
    counts = torch.tensor([(b + page - 1) // page for _, b in n])
    n_pages = int(counts.sum()) + 3
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).int()
    table = torch.zeros(c["seqs"], each, dtype=torch.int32)
    table[torch.arange(each)[None, :] < counts[:, None]] = order[:int(counts.sum())]
    normal = lambda *shape: torch.randn(*shape, generator=gen, device=DEVICE)       # noqa: E731
    chunk = 64 * _token_bytes(c)
    s = {"case": c, "table": table.to(DEVICE), "new": torch.tensor([a for a, _ in n], device=DEVICE), "rows": rows,
         "start": torch.tensor([0] + [sum(a for a, _ in n[:i + 1]) for i in range(len(n))], dtype=torch.int32, device=DEVICE),
         "len": torch.tensor([b for _, b in n], dtype=torch.int32, device=DEVICE), "max_new": max(a for a, _ in n), "max_len": longest}
    if c["op"] == "append":
        s["pages"] = torch.zeros(n_pages, kvh, page // 64, chunk, dtype=torch.uint8, device=DEVICE)
        s["q"], s["k"], s["v"] = normal(rows, c["heads"], h).mul(2).to(t), normal(rows, kvh, h).mul(2).to(t), normal(rows, kvh, h).to(t)
        s["gains"] = [1 + 0.1 * normal(h), 1 + 0.1 * normal(h)] if c["norm"] else [None, None]
        s["rope"] = _table(c, longest)
    else:
        k, v = normal(n_pages, kvh, page // 64, 64 * h), normal(n_pages, kvh, page // 64, 64 * h)
        kp, vp = (p.to(DEVICE) for p in _places(c["kv"], h))
        if c["kv"] == "fp8":
            (kc, ke), (vc, ve) = _quantise(k.view(-1, 64, h)), _quantise(v.view(-1, 64, h))
            parts = [kc.view(torch.uint8).view(k.shape)[..., kp], vc.view(torch.uint8).view(v.shape)[..., vp],
                     (ke + 127).to(torch.uint8).view(*k.shape[:3], 64), (ve + 127).to(torch.uint8).view(*k.shape[:3], 64)]
        else:
            tk = TYPES[c["kv"]]
            parts = [k.to(tk)[..., kp].view(torch.uint8), v.to(tk)[..., vp].view(torch.uint8)]
        s["pages"] = torch.cat(parts, -1).contiguous()
        s["q"] = normal(rows, c["heads"], h).mul(1.5).to(t) if c["op"] == "attend" else None
    s["k_rows"], s["v_rows"] = (torch.empty(rows, kvh, h, dtype=t, device=DEVICE) for _ in range(2)) if c["op"] != "attend" else (None, None)
    s["out"] = torch.empty_like(s["q"]) if s["q"] is not None else None
    if own:
        import paper_2410_01028_amd as asd
        types = {"f32": asd.DT_F32, "bf16": asd.DT_BF16, "fp8": asd.DT_FP8}
        s["cache"] = asd.KVCache(s["pages"], c["heads"], kvh, h, page, dtype=types[c["dtype"]], kv_dtype=types[c["kv"]])
        s["batch"] = asd.KVBatch(s["table"], s["start"], s["len"], n_rows=rows, max_new=s["max_new"], max_len=longest)
    return s


def run(s):
    c = s["case"]
    if own:
        cache, batch = s["cache"], s["batch"]
        if c["op"] == "attend":
            return cache.attend(batch, s["q"], out=s["out"])
        if c["op"] == "append":
            cache.append(batch, s["q"], s["k"], s["v"], q_out=s["out"], rope=s["rope"], rot_dim=c["rot"], interleaved=c["inter"],
                         q_gain=s["gains"][0], k_gain=s["gains"][1], eps=1e-5)
        cache.read(batch, k_out=s["k_rows"], v_out=s["v_rows"])
        return {"q": s["out"], "k": s["k_rows"], "v": s["v_rows"]}
    t = TYPES[c["dtype"]]
    if c["op"] == "append":
        pos = _positions(s)
        q = _rotate(c, _norm(s["q"].float(), s["gains"][0]), s["rope"][pos])
        k = _rotate(c, _norm(s["k"].float(), s["gains"][1]), s["rope"][pos])
        return {"q": q.to(t), "k": _held(c, k).to(t), "v": _held(c, s["v"].float()).to(t)}
    k, v = _dense(s)
    if c["op"] == "read":
        seq, pos = _sequence(s), _positions(s)
        return {"q": None, "k": k[seq, pos].to(t), "v": v[seq, pos].to(t)}
    # all sequences padded to the longest: rows [seq, KV head, new row x head of the group, dim]
    h, group, seqs, new = c["dim"], c["heads"] // c["kv_heads"], c["seqs"], s["max_new"]
    i, key = torch.arange(new, device=DEVICE), torch.arange(k.shape[1], device=DEVICE)
    at = (s["start"][:-1, None] + i).clamp(max=s["rows"] - 1)
    q = s["q"].float()[at].view(seqs, new, c["kv_heads"], group, h).permute(0, 2, 1, 3, 4).reshape(seqs, c["kv_heads"], new * group, h)
    score = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) / math.sqrt(h)
    last = (s["len"] - s["new"])[:, None] + i
    hidden = key > torch.minimum(last, s["len"][:, None] - 1)[..., None]
    score = score.view(seqs, c["kv_heads"], new, group, -1).masked_fill_(hidden[:, None, :, None, :], -math.inf)
    p = torch.exp(score.sub_(score.amax(-1, keepdim=True)))
    p = p.div_(p.sum(-1, keepdim=True)).view(seqs, c["kv_heads"], new * group, -1)
    o = torch.matmul(p, v.permute(0, 2, 1, 3).contiguous()).view(seqs, c["kv_heads"], new, group, h).permute(0, 2, 1, 3, 4)
    return o[_sequence(s), _positions(s) - (s["len"] - s["new"])[_sequence(s)]].reshape(s["rows"], c["heads"], h).to(t)


def _sequence(s):
    """The sequence of every packed row."""
    return torch.repeat_interleave(torch.arange(s["new"].numel(), device=DEVICE), s["new"], output_size=s["rows"])


def _positions(s):
    seq = _sequence(s)
    return torch.arange(s["rows"], device=DEVICE) - s["start"][seq] + (s["len"] - s["new"])[seq]


def _norm(x, gain):
    return x if gain is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5) * gain


def _rotate(c, x, cs):
    n = c["rot"]
    a, b = (x[..., 0:n:2], x[..., 1:n:2]) if c["inter"] else (x[..., :n // 2], x[..., n // 2:n])
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if c["inter"] else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., n:]], -1)


def _held(c, x):
    """The values that the cache holds of x."""
    if c["kv"] != "fp8":
        return x.to(TYPES[c["kv"]])
    code, e = _quantise(x)
    return torch.ldexp(code.float(), e)


def _dense(s):
    """K and V of every sequence, padded to whole pages of the longest: [seq, token, KV head, dim] in 32 bits; zeros behind its end."""
    c, h = s["case"], s["case"]["dim"]
    pages = s["pages"][s["table"].long()].permute(0, 2, 1, 3, 4).flatten(2, 3)      # [seq, KV head, chunk, bytes]
    kp, vp = (torch.argsort(p.to(DEVICE)) for p in _places(c["kv"], h))
    n = 64 * h * (_token_bytes(c) - (2 if c["kv"] == "fp8" else 0)) // (2 * h)
    kind = torch.float8_e4m3fn if c["kv"] == "fp8" else TYPES[c["kv"]]
    out = [pages[..., :n].contiguous().view(kind).float()[..., kp], pages[..., n:2 * n].contiguous().view(kind).float()[..., vp]]
    out = [x.view(*x.shape[:3], 64, h) for x in out]
    if c["kv"] == "fp8":
        out = [torch.ldexp(x, pages[..., 2 * n + 64 * i:2 * n + 64 * i + 64, None].int() - 127) for i, x in enumerate(out)]
    out = [x.flatten(2, 3).permute(0, 2, 1, 3) for x in out]
    past = torch.arange(out[0].shape[1], device=DEVICE) >= s["len"][:, None]
    return [x.masked_fill(past[..., None, None], 0.0) for x in out]


def exact(c, seed):
    s, n, h = prepare(c, seed), lens(c), c["dim"]

    def stored(x):          # nearest e4m3 number times the power of two, by its spacing
        if c["kv"] != "fp8":
            return x.to(TYPES[c["kv"]])
        top = x.abs().amax(-1, keepdim=True)
        unit = torch.exp2(torch.ceil(torch.log2((top / 448).clamp(min=2.0 ** -100))))
        y = x / unit
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        return torch.round(y / step) * step * unit

    if c["op"] == "append":
        def turned(x, gain):
            x = x.double()
            if gain is not None:
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / h + 1e-5) * gain.double()
            pos = torch.cat([torch.arange(b - a, b, dtype=torch.float64, device=DEVICE) for a, b in n])
            r, out = c["rot"], x.clone()
            for j in range(r // 2):
                # the angle's cosine and sine are inputs: the table's 32-bit values
                cos, sin = s["rope"][pos.long(), j].double().unbind(-1)
                u, w = (2 * j, 2 * j + 1) if c["inter"] else (j, j + r // 2)
                out[..., u] = x[..., u] * cos[:, None] - x[..., w] * sin[:, None]
                out[..., w] = x[..., w] * cos[:, None] + x[..., u] * sin[:, None]
            return out
        return {"q": turned(s["q"], s["gains"][0]), "k": stored(turned(s["k"], s["gains"][1])).double(), "v": stored(s["v"].double()).double()}
    page, group = c["page"], c["heads"] // c["kv_heads"]
    kp, vp = (p.to(DEVICE) for p in _places(c["kv"], h))
    width = {"f32": 4, "bf16": 2, "fp8": 1}[c["kv"]] * 64 * h
    outs, k_rows, v_rows = [], [], []
    for i, (new, total) in enumerate(n):
        blocks = s["pages"][s["table"][i, :(total + page - 1) // page].long()]       # [page, KV head, chunk, bytes]
        both = []
        for at, place in ((0, kp), (1, vp)):
            raw = blocks[..., at * width:(at + 1) * width].contiguous().view(torch.float8_e4m3fn if c["kv"] == "fp8" else TYPES[c["kv"]])
            x = torch.empty(*blocks.shape[:3], 64 * h, dtype=torch.float64, device=DEVICE)
            x[..., place] = raw.double()
            x = x.view(*blocks.shape[:3], 64, h)
            if c["kv"] == "fp8":
                x = x * torch.exp2(blocks[..., 2 * width + 64 * at:2 * width + 64 * at + 64].double() - 127)[..., None]
            both.append(x.permute(1, 0, 2, 3, 4).reshape(c["kv_heads"], -1, h)[:, :total])
        if c["op"] == "read":
            k_rows.append(both[0][:, total - new:].transpose(0, 1))
            v_rows.append(both[1][:, total - new:].transpose(0, 1))
            continue
        at = int(s["start"][i])
        hidden = torch.arange(total, device=DEVICE) > torch.arange(total - new, total, device=DEVICE)[:, None]
        heads = []
        for head in range(c["heads"]):
            k, v = both[0][head // group], both[1][head // group]
            z = (s["q"][at:at + new, head].double() @ k.T) / h ** 0.5
            heads.append(torch.softmax(z.masked_fill(hidden, -math.inf), -1) @ v)
        outs.append(torch.stack(heads, 1))
    return torch.cat(outs) if c["op"] == "attend" else {"q": None, "k": torch.cat(k_rows), "v": torch.cat(v_rows)}
