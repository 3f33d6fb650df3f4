"""Attention of sequences that begin with the same tokens (KVCache.attend_shared) against 64 bits; tolerances: kv_spans_reference.py.

`wide`: page tables with room for long sequences (entries that are no pages), for which the shared keys are read apart from the own ones.
"""
import math

import pytest
import torch

import paper_2410_01028_amd as asd
from kv_spans_reference import check, in_window
from test_gpu_kv_ops import COMBOS, DEV, Pool

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def widen(p):
    """Room for so many tokens that reading all of them for every sequence would be much."""
    each = asd.kv_page_bytes(p.cache.n_heads, p.cache.n_kv_heads, p.h, p.page, *p.cache._key[4:])
    n = len(p.lens)
    width = min(2 ** 24 // p.page, (2 ** 28 // n + each - 1) // each + 1)
    p.d_table = torch.cat([p.d_table, torch.full((n, max(0, width - p.d_table.shape[1])), -1, dtype=torch.int32, device=DEV)], 1).contiguous()
    p.cap = p.d_table.shape[1] * p.page


class Family:
    """Groups of sequences: (shared tokens, [(new rows, tokens) of its sequences]).  A group's first sequence holds the shared tokens; the others have pages of their
    own from the one on in which these end, with nothing but their own tokens written there."""

    def __init__(self, dtype, kv, heads, kv_heads, h, page, groups, seed=0, spread=0, max_len=None, wide=False):
        self.news, self.total = [n for _, g in groups for n, _ in g], [t for _, g in groups for _, t in g]
        self.shared, self.first = [s for s, g in groups for _ in g], []
        for _, g in groups:
            self.first += [len(self.first)] * len(g)
        p = self.p = Pool(dtype, kv, heads, kv_heads, h, page, list(zip(self.news, self.total)), seed=seed, max_len=max_len)
        if wide:
            widen(p)
        for i, f in enumerate(self.first):
            if f != i:
                p.d_table[i, :self.shared[i] // page] = p.d_table[f, :self.shared[i] // page]
                p.d_table[i, (self.total[i] + page - 1) // page:] = -1
        own = [t if i == f else max(0, t - s) for i, (f, s, t) in enumerate(zip(self.first, self.shared, self.total))]
        k, v = (p.normal(sum(own), kv_heads, h) for _ in range(2))
        if spread:
            for j, at in enumerate(range(0, sum(own), spread)):
                v[at, j % kv_heads, (3 * j) % h] = (math.nan, math.inf, -math.inf)[j % 3]
        written = p.batch(own, self.total)
        p.cache.append(written, None, k, v)
        k, v = (list(torch.split(x, own)) for x in p.cache.read(written))
        written.check()
        for i, f in enumerate(self.first):
            if f != i:
                k[i], v[i] = (torch.cat([x[f][:self.shared[i]], x[i]]) for x in (k, v))
        self.k, self.v = k, v
        self.start = [0]
        for _, g in groups:
            self.start.append(self.start[-1] + len(g))
        self.groups = asd.KVGroups(i32(self.start), i32([s for s, _ in groups]))

    def check(self, q, out, lens=None, scale=None):
        at = 0
        for i, (n, t) in enumerate(zip(self.news, lens or self.total)):
            if n:
                pos = torch.arange(t - n, t, device=DEV)
                check(self.p.dtype, q[at:at + n], out[at:at + n], self.k[i][:t], self.v[i][:t], in_window(pos, t, 2 ** 30, 0), scale or self.p.h ** -0.5, f"sequence {i}")
            at += n


FAMILIES = {
    "samples": [(130, [(1, 131), (1, 140), (1, 300), (1, 131)])],
    "drafts": [(700, [(5, 705)] * 5), (64, [(5, 80), (3, 67)])],
    "requests": [(333, [(70, 403), (1, 340), (0, 350), (33, 400)]), (128, [(64, 192), (20, 148), (130, 700)]), (1, [(9, 10), (4, 200)])],
    "alone": [(0, [(1, 5), (3, 70)]), (65, [(2, 90)]), (64, [(1, 65), (1, 1000)]), (7, []), (1000, [(1, 1001)])],
    "one group of all": [(2000, [(1 + i % 3, 2003 + 17 * i) for i in range(37)])],
    "not behind the shared tokens": [(100, [(100, 100), (1, 101), (2, 102)]), (64, [(3, 64), (5, 69), (1, 65)])],
}


@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
@pytest.mark.parametrize("dtype,kv", COMBOS)
@pytest.mark.parametrize("kind", list(FAMILIES))
@pytest.mark.parametrize("h,heads,kv_heads,page", [(128, 8, 1, 64), (128, 4, 4, 192), (64, 15, 5, 64), (32, 6, 2, 128)])
def test_families(dtype, kv, kind, h, heads, kv_heads, page, wide):
    f = Family(dtype, kv, heads, kv_heads, h, page, FAMILIES[kind], seed=h, wide=wide)
    rows = sum(f.news)
    q = f.p.normal(rows + 2, heads + 3, h, scale=2.0)[:, 1:heads + 1]
    out = torch.full((rows + 2, heads, h), 7.0, dtype=f.p.t, device=DEV)
    b = f.p.batch(f.news, f.total, extra=2)
    f.p.cache.attend_shared(b, f.groups, q, out=out)
    b.check()
    assert bool((out[rows:] == 7.0).all())
    f.check(q, out)


@pytest.mark.parametrize("dtype,kv", COMBOS)
@pytest.mark.parametrize("h,heads,kv_heads,groups", [(128, 64, 8, [(1000, [(1 + i % 5, 1007 + 11 * i) for i in range(20)]), (2111, [(3, 2114)] * 9)]),
                                                     (64, 40, 40, [(1500, [(1, 1501)] * 3 + [(4, 1700)] * 20)]), (64, 64, 4, [(65, [(1, 66)]), (3000, [(2, 3002 + i) for i in range(70)])])])
def test_rows_of_many_sequences_share_a_chunk(dtype, kv, h, heads, kv_heads, groups):
    """Groups whose rows fill tiles of 128 that go over the borders of sequences."""
    f = Family(dtype, kv, heads, kv_heads, h, 64, groups, seed=h, wide=True, spread=1013)
    q = f.p.normal(sum(f.news), heads, h, scale=2.0)
    b = f.p.batch(f.news, f.total)
    assert f.p.cache.attend_shared_workspace(b, f.groups) > 0
    out = f.p.cache.attend_shared(b, f.groups, q)
    b.check()
    f.check(q, out)


@pytest.mark.parametrize("kv", ["fp8", "bf16"])
@pytest.mark.parametrize("h,heads,kv_heads,page", [(128, 40, 40, 64), (128, 64, 8, 192), (64, 64, 8, 64)])
def test_many_rows(kv, h, heads, kv_heads, page):
    """Groups and sequences whose tiles fill the card."""
    f = Family("bf16", kv, heads, kv_heads, h, page, [(1000, [(64, 1064), (70, 1333), (1, 1020), (130, 1200)]), (333, [(0, 340), (200, 533), (17, 350), (2, 900)]),
                                                      (190, [(30, 220)] * 9)], seed=h)
    q = f.p.normal(sum(f.news) + 3, heads + 2, h, scale=2.0)[:, 1:heads + 1]
    out = torch.full((sum(f.news) + 3, heads, h), 7.0, dtype=f.p.t, device=DEV)
    b = f.p.batch(f.news, f.total, extra=3)
    f.p.cache.attend_shared(b, f.groups, q, out=out)
    b.check()
    assert bool((out[sum(f.news):] == 7.0).all())
    f.check(q, out)


@pytest.mark.parametrize("kv", ["fp8", "bf16"])
@pytest.mark.parametrize("groups", [[(20000, [(1, 20001 + 9 * i) for i in range(20)])], [(5000, [(6, 5006)] * 3), (64, [(1, 9000), (2, 70)])],
                                    [(9000, [(40, 9040), (1, 9001), (90, 12000)])]], ids=["tokens", "drafts and a long one", "chunks"])
def test_long_beginnings(kv, groups):
    """Shared and own keys that are cut into runs; more pages than a wave holds at a time."""
    f = Family("bf16", kv, 16, 2, 128, 64, groups, seed=3)
    q = f.p.normal(sum(f.news), 16, 128, scale=2.0)
    b = f.p.batch(f.news, f.total)
    out = f.p.cache.attend_shared(b, f.groups, q)
    b.check()
    f.check(q, out)


@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
@pytest.mark.parametrize("dtype,kv", COMBOS)
@pytest.mark.parametrize("kv_heads,kind", [(2, "samples"), (2, "drafts"), (2, "requests"), (64, "requests")])
def test_values_that_are_not_finite_stay_where_they_are_seen(dtype, kv, kv_heads, kind, wide):
    f = Family(dtype, kv, 2 * kv_heads, kv_heads, 64, 64, FAMILIES[kind], seed=2, spread=23, wide=wide)
    q = f.p.normal(sum(f.news), 2 * kv_heads, 64)
    b = f.p.batch(f.news, f.total)
    out = f.p.cache.attend_shared(b, f.groups, q)
    b.check()
    f.check(q, out)


@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
def test_more_groups_and_sequences_than_a_wave_looks_at(wide):
    groups = [((g * 37) % 200, [(1 + (g + i) % 2, (g * 37) % 200 + 2 + (i * 13) % 90) for i in range(g % 6)]) for g in range(150)]
    f = Family("bf16", "fp8", 4, 2, 64, 64, groups, seed=4, wide=wide)
    assert len(f.news) > 2 * len(groups)
    q = f.p.normal(sum(f.news), 4, 64)
    b = f.p.batch(f.news, f.total)
    out = f.p.cache.attend_shared(b, f.groups, q)
    b.check()
    f.check(q, out)


@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
def test_one_group_of_more_sequences_than_a_wave_looks_at(wide):
    f = Family("bf16", "bf16", 8, 2, 64, 64, [(70, [(1, 71)] * 3), (500, [(1, 501 + i) for i in range(200)]), (90, [(2, 200)] * 70)], seed=5, wide=wide)
    q = f.p.normal(sum(f.news), 8, 64)
    b = f.p.batch(f.news, f.total)
    out = f.p.cache.attend_shared(b, f.groups, q)
    b.check()
    f.check(q, out)


@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
def test_sequences_in_no_group(wide):
    """Groups of a few of the sequences: the others in front, between and behind take their own pages."""
    f = Family("bf16", "fp8", 8, 2, 64, 64, [(100, [(1, 130)]), (200, [(2, 202), (1, 300)]), (50, [(3, 80)]), (64, [(1, 90), (1, 70)])], seed=6, wide=wide)
    q = f.p.normal(sum(f.news), 8, 64)
    b = f.p.batch(f.news, f.total)
    for start, shared in (([1, 3], [200]), ([1, 3, 3], [200, 9]), ([1, 3, 3, 3], [200, 9, 7]), ([1, 3, 4, 6], [200, 50, 64])):
        out = f.p.cache.attend_shared(b, asd.KVGroups(i32(start), i32(shared)), q)
        b.check()
        rows = slice(1, 4)
        at = 1
        for i in (1, 2):
            n, t = f.news[i], f.total[i]
            check("bf16", q[at:at + n], out[at:at + n], f.k[i], f.v[i], in_window(torch.arange(t - n, t, device=DEV), t, 2 ** 30, 0), 0.125, f"sequence {i}")
            at += n
        assert bool(out[rows].isfinite().all())


@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
def test_rows_that_share_nothing_beside_others_and_answers_in_place(wide):
    """A group of sequences some of which do not reach behind the shared tokens, one whose first sequence does not hold them; the answer takes the queries' place, twice over: the
    same bits."""
    lens = [(2, 900), (1, 700), (1, 901), (5, 640), (2, 1000), (1, 100), (1, 800), (2, 650)]
    p = Pool("bf16", "fp8", 64, 8, 64, 64, lens, seed=15)
    if wide:
        widen(p)
    k, v = p.fill()
    p.d_table[1:5, :10] = p.d_table[0, :10]
    k, v = ([x[0]] + [torch.cat([x[0][:640], y[640:]]) for y in x[1:5]] + list(x[5:]) for x in (k, v))
    news, total = [a for a, _ in lens], [b for _, b in lens]
    b, groups = p.batch(news, total), asd.KVGroups(i32([0, 5, 8]), i32([640, 640]))
    q = p.normal(sum(news), 64, 64, scale=2.0)
    apart = p.cache.attend_shared(b, groups, q)
    at = 0
    for i, (n, t) in enumerate(lens):
        check("bf16", q[at:at + n], apart[at:at + n], k[i], v[i], in_window(torch.arange(t - n, t, device=DEV), t, 2 ** 30, 0), 0.125, f"sequence {i}")
        at += n
    for _ in range(4):
        mine = q.clone()
        assert p.cache.attend_shared(b, groups, mine, out=mine) is mine
        assert torch.equal(mine, apart)
    b.check()


BAD = {"descends": ([0, 4, 2, 6], [130, 130, 130]), "begins in front": ([-3, 2, 4, 6], [130, 130, 130]), "ends behind": ([0, 2, 4, 2 ** 31 - 1], [130, 130, 130]),
       "claimed twice": ([0, 6, 0, 6], [130, 130, 130]), "far away": ([2 ** 31 - 1, -2 ** 31, 2, 4], [130, 130, 130]), "lengths": ([0, 2, 4, 6], [-5, 2 ** 31 - 1, 130])}


@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
@pytest.mark.parametrize("dtype,kv", [("bf16", "fp8"), ("f32", "f32")])
@pytest.mark.parametrize("kind", list(BAD))
def test_groups_out_of_range_are_cut_and_reported(kind, dtype, kv, wide):
    """Sequences that hold all their tokens in pages of their own: whatever the groups say, each sequence's answer is that of its tokens."""
    lens = [(1, 200), (2, 300), (1, 131), (3, 400), (1, 150), (2, 170)]
    p = Pool(dtype, kv, 8, 2, 64, 64, lens, seed=7)
    if wide:
        widen(p)
    news, total = [a for a, _ in lens], [b for _, b in lens]
    k, v = p.normal(400, 2, 64), p.normal(400, 2, 64)
    own = [p.normal(300, 2, 64) for _ in range(12)]
    ks, vs = ([torch.cat([x[:130], y])[:t] for y, t in zip(ys, total)] for x, ys in ((k, own[:6]), (v, own[6:])))
    whole = p.batch(total, total)
    p.cache.append(whole, None, torch.cat(ks), torch.cat(vs))
    ks, vs = (torch.split(x, total) for x in p.cache.read(whole))
    q, b = p.normal(sum(news), 8, 64), p.batch(news, total)
    out = p.cache.attend_shared(b, asd.KVGroups(i32(BAD[kind][0]), i32(BAD[kind][1])), q)
    with pytest.raises(asd.AsdError, match="groups"):
        b.check()
    at = 0
    for i, (n, t) in enumerate(lens):
        check(dtype, q[at:at + n], out[at:at + n], ks[i], vs[i], in_window(torch.arange(t - n, t, device=DEV), t, 2 ** 30, 0), 0.125, f"sequence {i}")
        at += n


@pytest.mark.parametrize("start,lens", [([0, 3, 1, 6, 8], [200, 210, 220, 230]), ([0, 2, 4, 6, 2 ** 31 - 1], [200, 200, 200, 200]), ([-9, 2, 4, 6, 8], [200, 200, 200, 200]),
                                        ([0, 8, 0, 8, 8], [200, 200, 200, 200]), ([0, 2, 4, 6, 8], [2 ** 31 - 1, 1, -3, 200]), ([5, 4, 3, 2, 1], [200, 200, 200, 200])])
@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
def test_rows_out_of_range_are_cut_and_reported(start, lens, wide):
    """Rows that are claimed twice, cut or out of range beside groups: every answer is finite, rows that belong to no sequence stay as they are."""
    f = Family("bf16", "fp8", 8, 2, 64, 64, [(130, [(2, 200), (2, 200)]), (64, [(2, 200), (2, 200)])], seed=8, wide=wide)
    b = asd.KVBatch(f.p.d_table, i32(start), i32(lens), 8, 3, f.p.cap if wide else 200)
    q = f.p.normal(8, 8, 64)
    ref = f.p.cache.attend(b, q, out=torch.full_like(q, 7.0))
    out = f.p.cache.attend_shared(b, f.groups, q, out=torch.full_like(q, 7.0))
    with pytest.raises(asd.AsdError, match="rows or lengths"):
        b.check()
    assert torch.equal((out == 7.0).all(-1), (ref == 7.0).all(-1))


@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
def test_pages_out_of_range_are_hidden_and_reported(wide):
    f = Family("bf16", "bf16", 4, 2, 64, 64, [(200, [(1, 201), (2, 300), (1, 270)])], seed=9, wide=wide)
    q = f.p.normal(4, 4, 64)
    b = f.p.batch(f.news, f.total)
    for seq, page, hidden in ((0, 1, [0, 1, 2]), (1, 4, [1])):
        keep = f.p.d_table[seq, page].clone()
        for bad in (-1, f.p.cache.n_pages):
            f.p.d_table[seq, page] = bad
            out = f.p.cache.attend_shared(b, f.groups, q)
            with pytest.raises(asd.AsdError, match="pages"):
                b.check()
            at = 0
            for i, (n, t) in enumerate(zip(f.news, f.total)):
                seen = in_window(torch.arange(t - n, t, device=DEV), t, 2 ** 30, 0)
                if i in hidden:
                    seen[:, page * 64:page * 64 + 64] = False
                check("bf16", q[at:at + n], out[at:at + n], f.k[i], f.v[i], seen, 0.125, f"sequence {i}")
                at += n
        f.p.d_table[seq, page] = keep


@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
def test_a_fork_inside_a_page_goes_on_by_itself(wide):
    """A conversation is continued three ways: each way writes its own tokens from inside the page in which the common ones end, attends, and grows; the common
    tokens stay as they are.  In the end drafts for all of them are verified together."""
    h, heads, kv_heads, common = 64, 8, 2, 100
    p = Pool("bf16", "fp8", heads, kv_heads, h, 64, [(common, 300), (1, 300), (1, 300)], seed=10)
    if wide:
        widen(p)
    p.d_table[1:, :1] = p.d_table[0, :1]
    k, v = [p.normal(common, kv_heads, h)], [p.normal(common, kv_heads, h)]
    prompt = p.batch([common, 0, 0], [common, 0, 0])
    p.cache.append(prompt, None, k[0], v[0])
    k, v = ([x[:common]] * 3 for x in p.cache.read(prompt))
    groups = asd.KVGroups(i32([0, 3]), i32([common]))
    lens = [common] * 3
    for step, news in enumerate(([1, 1, 1], [1, 1, 1], [3, 1, 2], [5, 5, 5], [40, 70, 33])):
        lens = [t + n for t, n in zip(lens, news)]
        b = p.batch(news, lens)
        q, kn, vn = p.normal(sum(news), heads, h), p.normal(sum(news), kv_heads, h), p.normal(sum(news), kv_heads, h)
        p.cache.append(b, None, kn, vn)
        for x, got in zip((k, v), p.cache.read(b)):
            x[:] = [torch.cat([a, n]) for a, n in zip(x, torch.split(got, news))]
        out = p.cache.attend_shared(b, groups, q)
        b.check()
        at = 0
        for i, (n, t) in enumerate(zip(news, lens)):
            check("bf16", q[at:at + n], out[at:at + n], k[i], v[i], in_window(torch.arange(t - n, t, device=DEV), t, 2 ** 30, 0), h ** -0.5, f"step {step}, sequence {i}")
            at += n


@pytest.mark.parametrize("kind,wide", [("tokens", False), ("tokens", True), ("drafts", False), ("drafts", True), ("many", False)])
def test_a_captured_call_follows_lengths_and_groups(kind, wide):
    """Captured once, replayed with other lengths, groups and shared tokens, with eager work between: the eager call's bits; the answer in the queries' place."""
    news, heads, kv_heads = {"tokens": ([1] * 6, 16, 2), "drafts": ([6, 5, 1, 5, 2, 6], 8, 2), "many": ([130, 70, 1, 30, 40, 90], 64, 64)}[kind]
    longest = 2500
    p = Pool("bf16", "fp8", heads, kv_heads, 64, 64, [(n, longest) for n in news], seed=13)
    k, v = p.fill()
    if wide:
        widen(p)
    p.d_table[1:, :15] = p.d_table[0, :15]
    k, v = ([torch.cat([x[0][:960], y[960:]]) for y in x] for x in (k, v))
    b, groups = p.batch(news, news), asd.KVGroups(i32([0, 6, 6]), i32([0, 0]))
    q = p.normal(sum(news), heads, 64)
    ws = torch.empty(max(p.cache.attend_shared_workspace(b, groups), 256), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.cache.attend_shared(b, groups, q, out=q, workspace=ws)
    for lens, start, shared in (([longest] * 6, [0, 6, 6], [960, 0]), ([1200, 1300, 1000, 1150, 1100, 2500], [0, 3, 6], [900, 64]), (news, [0, 6, 6], [960, 0]),
                                ([1100] * 6, [0, 2, 6], [0, 700]), ([longest] * 6, [1, 4, 4], [960, 0])):
        b.kv_len.copy_(torch.tensor(lens))
        groups.group_start.copy_(torch.tensor(start)), groups.shared_len.copy_(torch.tensor(shared))
        rows = p.normal(sum(news), heads, 64)
        q.copy_(rows)
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        at = 0
        for i, (n, t) in enumerate(zip(news, lens)):
            check("bf16", rows[at:at + n], q[at:at + n], k[i][:t], v[i][:t], in_window(torch.arange(t - n, t, device=DEV), t, 2 ** 30, 0), 0.125, f"sequence {i}")
            at += n
        assert torch.equal(q, p.cache.attend_shared(b, groups, rows))
    b.check()


def test_two_calls_at_once_on_streams_of_their_own():
    f = Family("bf16", "fp8", 16, 2, 128, 64, [(3000, [(5, 3005)] * 4)], seed=14)
    b = [f.p.batch(f.news, f.total) for _ in range(2)]
    q = [f.p.normal(20, 16, 128) for _ in range(2)]
    want = [f.p.cache.attend_shared(x, f.groups, y) for x, y in zip(b, q)]
    out = [torch.empty_like(x) for x in q]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(8):
        for s, x, y, o in zip(streams, b, q, out):
            with torch.cuda.stream(s):
                f.p.cache.attend_shared(x, f.groups, y, out=o)
    torch.cuda.synchronize()
    for x, y, o, w in zip(b, q, out, want):
        x.check()
        assert torch.equal(o, w)
        f.check(y, o)


def test_refusals_of_the_binding():
    p = Pool("bf16", "fp8", 4, 2, 64, 64, [(2, 10)])
    p.fill()
    b, q, groups = p.batch([2], [10]), p.normal(2, 4, 64), asd.KVGroups(i32([0, 1]), i32([3]))
    for bad in ((i32([0, 1]), i32([3, 4])), (i32([0]), i32([])), (i32([0, 1]).long(), i32([3])), (i32([0, 1]).cpu(), i32([3])), (i32([0, 1]).cpu(), i32([3]).cpu()),
                (i32([[0, 1]]), i32([3])), (i32([0, 0, 1, 1])[::2], i32([3]))):
        with pytest.raises(asd.AsdError):
            asd.KVGroups(*bad)
    for bad in (q.float(), q[:1], q.cpu()):
        with pytest.raises(asd.AsdError):
            p.cache.attend_shared(b, groups, bad)
    with pytest.raises(asd.AsdError):
        p.cache.attend_shared(b, groups, q, workspace=torch.empty(256, dtype=torch.uint8))
    with pytest.raises(AttributeError):
        groups.shared_len = i32([4])
