"""Cases of two forms of attention over a paged cache of several sequences (`KVCache` in the Python binding).

  window   every sequence's new tokens attend to the last `window` tokens in front of them (themselves included) and to the first
           `sinks` tokens of the sequence, which stay visible: one token each (decoding), a few (verification of drafts), a chunk
           behind a long context, whole prompts.
  shared   sequences in groups that begin with the same tokens (samples of one prompt, drafts of one conversation, requests behind
           one system prompt): causal attention, the group's common keys read through the first member's pages.

Sequences share one pool of pages through a page table (pages in random order); rows of all sequences are packed one behind the
other.  Head counts and widths are those of the shapes in `asd_inputs.SHAPES` (tiny, 7b, 13b, 70b).
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEVICE = "cuda:0" if torch.cuda.is_available() else "cpu"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _case(name, op, dtype, kv, heads, kv_heads, dim, page, seqs, new, ctx, mix, window=0, sinks=0, groups=0, shared=0):
    """new: most new rows of a sequence; ctx: most tokens of a sequence with the new ones, and behind the shared ones (0: the new
    ones are all there is); mix: 0 for sequences (and groups) of one length, else the seed of their lengths; shared: most tokens
    that a group shares."""
    return {"name": name, "op": op, "dtype": dtype, "kv": kv, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page,
            "seqs": seqs, "new": new, "ctx": ctx, "mix": mix, "window": window, "sinks": sinks, "groups": groups, "shared": shared}


def listed():
    return [
        # the smallest call: one token of the small fp32 model behind 44 tokens
        _case("window-one", "window", "f32", "f32", 4, 4, 64, 64, 1, 1, 45, 0, window=32, sinks=4),
        # decoding of 48 conversations of 500 to 8192 tokens on the 70B heads
        _case("window-decode", "window", "bf16", "fp8", 64, 8, 128, 64, 48, 1, 8192, 3, window=1024, sinks=4),
        # one long conversation alone on the 7B heads, cache in bf16
        _case("window-alone", "window", "bf16", "bf16", 32, 32, 128, 256, 1, 1, 8192, 0, window=4096, sinks=4),
        # verification of four drafts and the token before them for eight sequences of the 13B heads
        _case("window-verify", "window", "bf16", "fp8", 40, 40, 128, 64, 8, 5, 4111, 11, window=500, sinks=1),
        # a chunk of 512 new tokens behind a long document, two requests, 70B heads
        _case("window-chunk", "window", "bf16", "fp8", 64, 8, 128, 64, 2, 512, 8707, 13, window=2048, sinks=4),
        # whole prompts of four requests on the 7B heads, cache in bf16
        _case("window-prompt", "window", "bf16", "bf16", 32, 32, 128, 64, 4, 4096, 0, 5, window=1024, sinks=4),
        # a small fp32 model: ragged chunks of three sequences, grouped heads, a short window and first tokens beyond a chunk of 64
        _case("window-f32", "window", "f32", "f32", 8, 2, 64, 64, 3, 61, 300, 17, window=37, sinks=70),
        # 64 answers to one long document, one token each, on the 70B heads
        _case("shared-decode", "shared", "bf16", "fp8", 64, 8, 128, 64, 64, 1, 300, 3, groups=1, shared=8005),
        # sixteen samples of a prompt on the 7B heads, cache in bf16
        _case("shared-samples", "shared", "bf16", "bf16", 32, 32, 128, 64, 16, 1, 512, 7, groups=1, shared=2048),
        # eight drafts of five tokens behind one conversation (13B heads), verified together
        _case("shared-drafts", "shared", "bf16", "fp8", 40, 40, 128, 64, 8, 5, 0, 0, groups=1, shared=1031),
        # 24 questions behind three system prompts on the 70B heads
        _case("shared-requests", "shared", "bf16", "fp8", 64, 8, 128, 64, 24, 130, 0, 9, groups=3, shared=4000),
        # a small fp32 model: seven sequences in two groups, ragged
        _case("shared-f32", "shared", "f32", "f32", 8, 2, 64, 64, 7, 9, 70, 19, groups=2, shared=150),
    ]


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / 1e15 * (8 if c["dtype"] == "f32" else 1))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["window", "shared"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        kv, dim = rng.choice([dtype, "fp8", "fp8"]), rng.choice([64, 128, 128])
        kv_heads, group = rng.choice([(1, 8), (2, 4), (4, 1), (5, 3), (8, 8), (8, 4), (32, 1), (40, 1)])
        wide = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))     # noqa: E731
        new = rng.choice([1, 1, wide(2, 16), wide(16, 2048 if op == "window" else 256)])
        seqs, mix, page = wide(1, 64), rng.randrange(0, 1000), rng.choice([64, 64, 128, 256])
        if op == "window":
            c = _case("", op, dtype, kv, kv_heads * group, kv_heads, dim, page, seqs, new, new + rng.choice([0, wide(1, 8192), wide(1, 8192)]), mix,
                      window=wide(1, 8192), sinks=rng.choice([0, 4, wide(1, 200)]))
        else:
            c = _case("", op, dtype, kv, kv_heads * group, kv_heads, dim, page, seqs, new, rng.choice([0, new + wide(1, 1024)]), mix,
                      groups=min(seqs, rng.choice([1, 1, wide(1, 12)])), shared=wide(1, 8192))
        # the most that the plain form of a batch takes: scores of all sequences padded to the longest, in 32 bits
        keys = min(c["ctx"], c["window"] + c["new"] + c["sinks"] + 128) if op == "window" else c["shared"] + max(c["ctx"], c["new"])
        if _cost(c) <= most and c["seqs"] * c["heads"] * c["new"] * keys < 2 ** 31 and c["seqs"] * keys * c["kv_heads"] * dim < 2 ** 30:
            del c["name"]
            return c


def groups(c):
    """(sequences, shared tokens) of every group, in order; the first shares most."""
    r, n = random.Random(c["mix"] + 1), max(c["groups"], 1)
    cuts = sorted(r.sample(range(1, c["seqs"]), n - 1)) if c["mix"] else [c["seqs"] * i // n for i in range(1, n)]
    return [(b - a, c["shared"] if not c["mix"] or a == 0 else r.randint((c["shared"] + 3) // 4, c["shared"]))
            for a, b in zip([0] + cuts, cuts + [c["seqs"]])]


def lens(c):
    """(new rows, tokens, shared tokens) of every sequence; the first is the longest."""
    r, out = random.Random(c["mix"]), []
    common = [s for n, s in groups(c) for _ in range(n)]
    for s in range(c["seqs"]):
        new = c["new"] if not c["mix"] or s == 0 else r.randint((c["new"] + 3) // 4, c["new"])
        most = max(c["ctx"], c["new"])
        total = new if not c["ctx"] else most if not c["mix"] or s == 0 else r.randint(max(new, most // 16), most)
        out.append((new, common[s] + total, common[s]))
    return out


def _token_bytes(c):
    """What a token and KV head take in the cache."""
    return 2 * c["dim"] * {"f32": 4, "bf16": 2, "fp8": 1}[c["kv"]] + (2 if c["kv"] == "fp8" else 0)


def _seen(c, pos):
    """Keys that a row at this position sees."""
    return pos + 1 if c["op"] == "shared" else min(pos + 1, c["window"] + min(c["sinks"], max(pos + 1 - c["window"], 0)))


def work(c):
    n, e = lens(c), 4 if c["dtype"] == "f32" else 2
    rows, seen = sum(a for a, _, _ in n), sum(_seen(c, p) for a, b, _ in n for p in range(b - a, b))
    if c["op"] == "shared":
        tokens = sum(s for _, s in groups(c)) + sum(b - s for _, b, s in n)
    else:
        tokens = sum(a - 1 + _seen(c, b - a) for a, b, _ in n)        # what the first row sees, and the rows behind it
    return {"bytes": rows * c["heads"] * 2 * c["dim"] * e + tokens * c["kv_heads"] * _token_bytes(c), "flops": 4 * c["dim"] * c["heads"] * seen}


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


def prepare(c, seed):
    gen = torch.Generator(DEVICE).manual_seed(seed)
    n, h, kvh, t, page = lens(c), c["dim"], c["kv_heads"], TYPES[c["dtype"]], c["page"]
    rows, longest = sum(a for a, _, _ in n), max(b for _, b, _ in n)
    # a sequence has pages of its own from the one on in which the shared tokens end, the group's first one all of its pages
    members, first = groups(c), []
    for size, _ in members:
        first += [len(first)] * size
    begin = [0 if first[i] == i else s // page for i, (_, _, s) in enumerate(n)]
    end = [(b + page - 1) // page for _, b, _ in n]
    n_pages = sum(end) - sum(begin) + 3
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).int()
    table, used = torch.zeros(c["seqs"], max(end), dtype=torch.int32), 0
    for i in range(c["seqs"]):
        table[i, :begin[i]] = table[first[i], :begin[i]]
        table[i, begin[i]:end[i]] = order[used:used + end[i] - begin[i]]
        used += end[i] - begin[i]
    normal = lambda *shape: torch.randn(*shape, generator=gen, device=DEVICE)       # noqa: E731
    k, v = normal(n_pages, kvh, page // 64, 64 * h), normal(n_pages, kvh, page // 64, 64 * h)
    kp, vp = (p.to(DEVICE) for p in _places(c["kv"], h))
    if c["kv"] == "fp8":
        (kc, ke), (vc, ve) = _quantise(k.view(-1, 64, h)), _quantise(v.view(-1, 64, h))
        parts = [kc.view(torch.uint8).view(k.shape)[..., kp], vc.view(torch.uint8).view(v.shape)[..., vp],
                 (ke + 127).to(torch.uint8).view(*k.shape[:3], 64), (ve + 127).to(torch.uint8).view(*k.shape[:3], 64)]
    else:
        tk = TYPES[c["kv"]]
        parts = [k.to(tk)[..., kp].view(torch.uint8), v.to(tk)[..., vp].view(torch.uint8)]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEVICE)              # noqa: E731
    s = {"case": c, "pages": torch.cat(parts, -1).contiguous(), "table": table.to(DEVICE), "rows": rows, "max_new": max(a for a, _, _ in n), "max_len": longest,
         "start": ints([sum(a for a, _, _ in n[:i]) for i in range(len(n) + 1)]), "len": ints([b for _, b, _ in n]), "new": ints([a for a, _, _ in n]),
         "group_start": ints([sum(size for size, _ in members[:i]) for i in range(len(members) + 1)]), "shared": ints([x for _, x in members]),
         "q": normal(rows, c["heads"], h).mul(1.5).to(t)}
    s["out"] = torch.empty_like(s["q"])
    if own:
        import paper_2410_01028_amd as asd
        types = {"f32": asd.DT_F32, "bf16": asd.DT_BF16, "fp8": asd.DT_FP8}
        s["cache"] = asd.KVCache(s["pages"], c["heads"], kvh, h, page, dtype=types[c["dtype"]], kv_dtype=types[c["kv"]])
        s["batch"] = asd.KVBatch(s["table"], s["start"], s["len"], n_rows=rows, max_new=s["max_new"], max_len=longest)
        s["groups"] = asd.KVGroups(s["group_start"], s["shared"]) if c["op"] == "shared" else None
    return s


def run(s):
    c = s["case"]
    if own:
        if c["op"] == "window":
            return s["cache"].attend_window(s["batch"], s["q"], window=c["window"], sinks=c["sinks"], out=s["out"])
        return s["cache"].attend_shared(s["batch"], s["groups"], s["q"], out=s["out"])
    return _window(s) if c["op"] == "window" else _shared(s)


def _padded(s):
    """Queries [seq, KV head, new row x head of the group, dim] of all sequences padded to the most rows, and the rows' positions [seq, new row]."""
    c = s["case"]
    i = torch.arange(s["max_new"], device=DEVICE)
    q = s["q"].float()[(s["start"][:-1, None] + i).clamp(max=s["rows"] - 1)]
    q = q.view(c["seqs"], s["max_new"], c["kv_heads"], -1, c["dim"]).permute(0, 2, 1, 3, 4).flatten(2, 3)
    return q, torch.minimum((s["len"] - s["new"])[:, None] + i, s["len"][:, None] - 1)


def _packed(s, o):
    """Rows [row, head, dim] out of [seq, KV head, new row x head of the group, dim]."""
    c = s["case"]
    o = o.view(c["seqs"], c["kv_heads"], s["max_new"], -1, c["dim"]).permute(0, 2, 1, 3, 4).flatten(2, 3)
    seq = torch.repeat_interleave(torch.arange(c["seqs"], device=DEVICE), s["new"], output_size=s["rows"])
    return o[seq, torch.arange(s["rows"], device=DEVICE) - s["start"][seq]].to(TYPES[c["dtype"]])


def _window(s):
    c = s["case"]
    q, pos = _padded(s)
    # the chunks of 64 tokens that hold the first tokens and the windows of all new rows
    first = (s["len"] - s["new"] - c["window"] + 1).clamp(min=0) // 64
    n_sink = (c["sinks"] + 63) // 64
    n_near = min((c["window"] + s["max_new"] - 2) // 64 + 2, (s["max_len"] + 63) // 64)
    near = first[:, None] + torch.arange(n_near, device=DEVICE)
    chunk = torch.cat([torch.arange(n_sink, device=DEVICE).expand(c["seqs"], -1), near], 1)
    k, v, key = _dense(s, s["table"], chunk)
    twice = torch.cat([torch.arange(n_sink, device=DEVICE) >= first[:, None], torch.zeros_like(near, dtype=torch.bool)], 1).repeat_interleave(64, 1)
    key = torch.where(twice | (key >= s["len"][:, None]), 2 ** 30, key)[:, None, :]
    seen = (key <= pos[..., None]) & ((key > pos[..., None] - c["window"]) | (key < c["sinks"]))
    v = v.masked_fill((key[:, 0] == 2 ** 30)[:, None, :, None], 0.0)
    score = torch.matmul(q, k.transpose(-1, -2).contiguous()) / math.sqrt(c["dim"])
    score.view(c["seqs"], c["kv_heads"], s["max_new"], -1, key.shape[-1]).masked_fill_(~seen[:, None, :, None, :], -math.inf)
    p = torch.exp(score.sub_(score.amax(-1, keepdim=True)))
    return _packed(s, torch.matmul(p.div_(p.sum(-1, keepdim=True)), v))


def _shared(s):
    c, h = s["case"], s["case"]["dim"]
    q, pos = _padded(s)
    size = [n for n, _ in groups(c)]
    common = torch.repeat_interleave(s["shared"], torch.tensor(size, device=DEVICE), output_size=c["seqs"])
    # each sequence's own keys, padded to the most
    n_own = (max(b - x // 64 * 64 for _, b, x in lens(c)) + 63) // 64
    k, v, key = _dense(s, s["table"], common[:, None] // 64 + torch.arange(n_own, device=DEVICE))
    gone = (key < common[:, None]) | (key >= s["len"][:, None])
    score = torch.matmul(q, k.transpose(-1, -2).contiguous()) / math.sqrt(h)
    hidden = gone[:, None, :] | (key[:, None, :] > pos[..., None])
    score.view(c["seqs"], c["kv_heads"], s["max_new"], -1, key.shape[-1]).masked_fill_(hidden[:, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score.sub_(top))
    total, o = p.sum(-1, keepdim=True), torch.matmul(p, v.masked_fill(gone[:, None, :, None], 0.0))
    # the shared keys, all rows of a group at once
    parts, at = [], 0
    for n, x in groups(c):
        k, v, _ = _dense(s, s["table"][at:at + 1], torch.arange((x + 63) // 64, device=DEVICE)[None])
        rows = q[at:at + n].transpose(0, 1).flatten(1, 2)                           # [KV head, all rows of the group, dim]
        z = torch.matmul(rows, k[0, :, :x].transpose(-1, -2).contiguous()) / math.sqrt(h)
        m = z.amax(-1, keepdim=True)
        z = torch.exp(z.sub_(m))
        parts.append([y.view(c["kv_heads"], n, -1, y.shape[-1]).transpose(0, 1) for y in (m, z.sum(-1, keepdim=True), torch.matmul(z, v[0, :, :x].contiguous()))])
        at += n
    m, z, x = (torch.cat(y) for y in zip(*parts))
    ref = torch.maximum(top, m)
    a, b = torch.exp(top - ref), torch.exp(m - ref)
    return _packed(s, (o * a + x * b) / (total * a + z * b))


def _dense(s, table, chunk):
    """K and V [seq, KV head, key, dim] in 32 bits of the chunks [seq, n] of 64 tokens of the sequences of these table rows, and the keys' positions [seq, key]."""
    c, h, per = s["case"], s["case"]["dim"], s["case"]["page"] // 64
    page = torch.gather(table.long(), 1, (chunk // per).clamp(max=table.shape[1] - 1))
    blocks = s["pages"].permute(0, 2, 1, 3)[page, chunk % per].transpose(1, 2)      # [seq, KV head, chunk, bytes]
    kp, vp = (torch.argsort(p.to(DEVICE)) for p in _places(c["kv"], h))
    n = 64 * h * (_token_bytes(c) - (2 if c["kv"] == "fp8" else 0)) // (2 * h)
    kind = torch.float8_e4m3fn if c["kv"] == "fp8" else TYPES[c["kv"]]
    out = [blocks[..., :n].contiguous().view(kind).float()[..., kp], blocks[..., n:2 * n].contiguous().view(kind).float()[..., vp]]
    out = [x.view(*x.shape[:3], 64, h) for x in out]
    if c["kv"] == "fp8":
        out = [torch.ldexp(x, blocks[..., 2 * n + 64 * i:2 * n + 64 * i + 64, None].int() - 127) for i, x in enumerate(out)]
    return [x.flatten(2, 3) for x in out] + [(chunk[..., None] * 64 + torch.arange(64, device=DEVICE)).flatten(1)]


def exact(c, seed):
    s, n, h, page, group = prepare(c, seed), lens(c), c["dim"], c["page"], c["heads"] // c["kv_heads"]
    kp, vp = (p.to(DEVICE) for p in _places(c["kv"], h))
    width = {"f32": 4, "bf16": 2, "fp8": 1}[c["kv"]] * 64 * h

    def sequence(i, tokens):
        """K and V [KV head, token, dim] of a sequence's first tokens through its own table row."""
        blocks, both = s["pages"][s["table"][i, :(tokens + page - 1) // page].long()], []
        for at, place in ((0, kp), (1, vp)):
            raw = blocks[..., at * width:(at + 1) * width].contiguous().view(torch.float8_e4m3fn if c["kv"] == "fp8" else TYPES[c["kv"]])
            x = torch.empty(*blocks.shape[:3], 64 * h, dtype=torch.float64, device=DEVICE)
            x[..., place] = raw.double()
            x = x.view(*blocks.shape[:3], 64, h)
            if c["kv"] == "fp8":
                x = x * torch.exp2(blocks[..., 2 * width + 64 * at:2 * width + 64 * at + 64].double() - 127)[..., None]
            both.append(x.permute(1, 0, 2, 3, 4).reshape(c["kv_heads"], -1, h)[:, :tokens])
        return both

    outs, row, leader = [], 0, 0
    begins = {sum(size for size, _ in groups(c)[:j]) for j in range(len(groups(c)))}
    for i, (new, total, common) in enumerate(n):
        k, v = sequence(i, total)
        if i in begins:
            leader = i
            front = sequence(i, common)
        if i != leader:
            k, v = torch.cat([front[0], k[:, common:]], 1), torch.cat([front[1], v[:, common:]], 1)
        p, j = torch.arange(total - new, total, device=DEVICE)[:, None], torch.arange(total, device=DEVICE)[None, :]
        hidden = j > p
        if c["op"] == "window":
            hidden = hidden | ((p - j >= c["window"]) & (j >= c["sinks"]))
        heads = []
        for x in range(c["kv_heads"]):
            q = s["q"][row:row + new, x * group:(x + 1) * group].double().transpose(0, 1).reshape(group * new, h)
            z = (q @ k[x].T / h ** 0.5).view(group, new, total).masked_fill(hidden, -math.inf)
            heads.append((torch.softmax(z, -1).view(group * new, total) @ v[x]).view(group, new, h).transpose(0, 1))
        outs.append(torch.cat(heads, 1))
        row += new
    return torch.cat(outs)
