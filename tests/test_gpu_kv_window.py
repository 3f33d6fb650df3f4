"""Attention with a sliding window and first tokens that stay visible (KVCache.attend_window) against 64 bits; tolerances: kv_spans_reference.py."""
import math

import pytest
import torch

import paper_2410_01028_amd as asd
from kv_spans_reference import check, in_window
from test_gpu_kv_ops import COMBOS, DEV, LENS, Pool

pytestmark = pytest.mark.gpu

KINDS = {
    "tokens": [(1, 1), (1, 63), (1, 64), (1, 65), (0, 7), (1, 257), (1, 1000), (1, 2500)],
    "drafts": [(5, 5), (3, 70), (5, 600), (1, 129), (4, 64)],
    "chunks": [(64, 64), (70, 333), (1, 20), (130, 1200)],
    "ragged": LENS,
}
SPANS = [(1, 0), (1, 1), (5, 3), (64, 64), (63, 4), (100, 130), (500, 4), (7, 200), (333, 0), (5000, 0), (2 ** 31 - 1, 2 ** 31 - 1)]


def check_window(p, news, lens, q, out, k, v, scale, window, sinks):
    at = 0
    for i, (n, length) in enumerate(zip(news, lens)):
        if n:
            pos = torch.arange(length - n, length, device=DEV)
            check(p.dtype, q[at:at + n], out[at:at + n], k[i][:length], v[i][:length], in_window(pos, length, window, sinks), scale, f"sequence {i}, window {window}, {sinks}")
        at += n


@pytest.mark.parametrize("dtype,kv", COMBOS)
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("h,heads,kv_heads,page", [(128, 8, 1, 64), (128, 4, 4, 192), (64, 15, 5, 64), (32, 6, 2, 128)])
def test_windows(dtype, kv, kind, h, heads, kv_heads, page):
    p = Pool(dtype, kv, heads, kv_heads, h, page, KINDS[kind], seed=h)
    k, v = p.fill()
    news, total = [a for a, _ in KINDS[kind]], [b for _, b in KINDS[kind]]
    rows = sum(news)
    q = p.normal(rows + 2, heads + 3, h, scale=2.0)[:, 1:heads + 1]
    b = p.batch(news, total, extra=2)
    for window, sinks in SPANS:
        out = torch.full((rows + 2, heads, h), 7.0, dtype=p.t, device=DEV)
        p.cache.attend_window(b, q, window, sinks, out=out)
        b.check()
        assert bool((out[rows:] == 7.0).all())
        check_window(p, news, total, q, out, k, v, h ** -0.5, window, sinks)


@pytest.mark.parametrize("kv", ["fp8", "bf16"])
@pytest.mark.parametrize("h,heads,kv_heads,page", [(128, 40, 40, 64), (128, 64, 8, 192), (64, 64, 8, 64), (64, 40, 40, 128)])
def test_many_rows(kv, h, heads, kv_heads, page):
    """Batches whose tiles fill the card: chunks, whole prompts, a single token and nothing among them."""
    news, total = [64, 70, 1, 130, 0, 200, 17, 2, 300], [64, 333, 20, 1200, 9, 200, 17, 2, 301]
    p = Pool("bf16", kv, heads, kv_heads, h, page, list(zip(news, total)), seed=h)
    k, v = p.fill()
    q = p.normal(sum(news) + 3, heads + 2, h, scale=2.0)[:, 1:heads + 1]
    b = p.batch(news, total, extra=3)
    for window, sinks in ((1, 0), (64, 4), (100, 70), (37, 64), (250, 1), (1000, 130), (5000, 0)):
        out = torch.full((sum(news) + 3, heads, h), 7.0, dtype=p.t, device=DEV)
        p.cache.attend_window(b, q, window, sinks, out=out)
        b.check()
        assert bool((out[sum(news):] == 7.0).all())
        check_window(p, news, total, q, out, k, v, h ** -0.5, window, sinks)


@pytest.mark.parametrize("kv", ["fp8", "bf16"])
def test_long_and_lopsided_batches(kv):
    """Windows that are cut into runs and joined: a token, a few rows, chunks; first tokens of many pages, and of more than a wave holds at a time."""
    for news, total in (((1, 1, 1, 1), (20000, 40, 1, 700)), ((6, 0, 2, 6), (9000, 40, 2, 7000)), ((150, 1, 90, 3), (6000, 40, 90, 2100)), ((300, 1, 90, 3), (9000, 40, 90, 2100))):
        p = Pool("bf16", kv, 8, 2, 128, 64, list(zip(news, total)), seed=3)
        k, v = p.fill()
        b = p.batch(news, total)
        q = p.normal(sum(news), 8, 128, scale=2.0)
        for window, sinks in ((4096, 4), (1500, 700), (3000, 5000), (64, 4200), (9000, 0)):
            out = p.cache.attend_window(b, q, window, sinks)
            b.check()
            check_window(p, news, total, q, out, k, v, 128 ** -0.5, window, sinks)


def test_a_window_that_reaches_everything_is_causal_attention():
    news, total = [64, 1, 5, 130], [64, 2500, 600, 1200]
    for dtype, kv in COMBOS:
        p = Pool(dtype, kv, 8, 2, 64, 64, list(zip(news, total)), seed=9)
        k, v = p.fill()
        b = p.batch(news, total)
        q = p.normal(sum(news), 8, 64)
        for window, sinks in ((2500, 0), (1, 2500), (2 ** 31 - 1, 7)):
            check_window(p, news, total, q, p.cache.attend_window(b, q, window, sinks), k, v, 0.125, 2500, 0)
        b.check()


@pytest.mark.parametrize("dtype,kv", COMBOS)
@pytest.mark.parametrize("news,kv_heads", [((40, 6, 90), 64), ((40, 6, 90), 2), ((5, 3, 4), 2), ((1, 6, 1), 2)], ids=["many rows", "chunks", "drafts", "tokens"])
def test_values_that_are_not_finite_stay_where_they_are_seen(dtype, kv, news, kv_heads):
    """Infinities and NaN in V and NaN in K at keys behind the window, among the first tokens, at the borders of both, and where all rows see them."""
    total, h = [400, 6, 330], 64
    p = Pool(dtype, kv, 2 * kv_heads, kv_heads, h, 64, list(zip(news, total)), seed=1)
    k, v = p.normal(sum(total), kv_heads, h), p.normal(sum(total), kv_heads, h)
    for i, key in enumerate((0, 3, 4, 63, 64, 100, 199, 200, 201, 239, 255, 256, 299, 300, 301, 320, 359, 360, 398, 399)):
        v[key, i % 2, 3 * i] = (math.nan, math.inf, -math.inf)[i % 3]
        if key < 330:
            v[406 + key, (i + 1) % 2, 63 - 3 * i] = (math.inf, math.nan, -math.inf)[i % 3]
    k[150, 0, 5] = k[406 + 70, 1, 5] = math.nan
    whole = p.batch(total, total)
    p.cache.append(whole, None, k, v)
    k, v = (torch.split(x, total) for x in p.cache.read(whole))
    b = p.batch(news, total)
    q = p.normal(sum(news), 2 * kv_heads, h)
    for window, sinks in ((100, 4), (200, 0), (64, 64), (130, 5), (20, 100)):
        out = p.cache.attend_window(b, q, window, sinks)
        b.check()
        check_window(p, news, total, q, out, k, v, h ** -0.5, window, sinks)


@pytest.mark.parametrize("kv", ["fp8", "bf16"])
def test_values_that_are_not_finite_in_runs_of_many_rows(kv):
    """Windows that are cut into runs, for tiles of many rows: at the first and last keys of the first tokens, of the windows and of chunks."""
    news, total = [300, 1, 90, 3], [9000, 40, 90, 2100]
    p = Pool("bf16", kv, 8, 2, 128, 256, list(zip(news, total)), seed=24)
    k, v = p.normal(sum(total), 2, 128), p.normal(sum(total), 2, 128)
    for i, key in enumerate((0, 63, 64, 1023, 1024, 2047, 3000, 4700, 4701, 4735, 4736, 5000, 5119, 8699, 8700, 8703, 8704, 8767, 8900, 8999)):
        v[key, i % 2, 3 * i] = (math.nan, math.inf, -math.inf)[i % 3]
    whole = p.batch(total, total)
    p.cache.append(whole, None, k, v)
    k, v = (torch.split(x, total) for x in p.cache.read(whole))
    b = p.batch(news, total)
    q = p.normal(sum(news), 8, 128)
    for window, sinks in ((4000, 64), (4000, 1000), (600, 1), (8000, 65)):
        out = p.cache.attend_window(b, q, window, sinks)
        b.check()
        check_window(p, news, total, q, out, k, v, 128 ** -0.5, window, sinks)


@pytest.mark.parametrize("dtype,kv", COMBOS)
@pytest.mark.parametrize("kind", ["tokens", "drafts", "chunks"])
def test_pages_behind_the_window_may_be_gone(dtype, kv, kind):
    """Pages that no row of the batch sees are not looked at: their entries in the table are anything.  One that is seen and missing is hidden and reported."""
    lens = [(n, t + 900) for n, t in KINDS[kind]]
    p = Pool(dtype, kv, 8, 2, 64, 64, lens, seed=5)
    k, v = p.fill()
    news, total = [a for a, _ in lens], [b for _, b in lens]
    b, q = p.batch(news, total), p.normal(sum(news), 8, 64)
    window, sinks = 200, 70
    want = p.cache.attend_window(b, q, window, sinks)
    for i, (n, t) in enumerate(lens):
        first = max(0, t - n - window + 1) // 64
        p.d_table[i, 2:max(2, first)] = torch.tensor([-1, 2 ** 31 - 1, p.cache.n_pages], dtype=torch.int32, device=DEV).repeat(30)[:max(0, first - 2)]
        p.d_table[i, (t + 63) // 64:] = -7
    got = p.cache.attend_window(b, q, window, sinks)
    b.check()
    assert torch.equal(got, want)
    check_window(p, news, total, q, got, k, v, 0.125, window, sinks)
    p.d_table[0, 0] = -1
    got = p.cache.attend_window(b, q, window, sinks)
    with pytest.raises(asd.AsdError, match="pages"):
        b.check()
    n, t = lens[0]
    seen = in_window(torch.arange(t - n, t, device=DEV), t, window, sinks)
    seen[:, :64] = False
    check(dtype, q[:n], got[:n], k[0][:t], v[0][:t], seen, 0.125, "a page of the first tokens is missing")
    assert torch.equal(got[n:], want[n:])


def test_more_sequences_than_a_wave_looks_at():
    lens = [(i % 3, 1 + (i * 37) % 450 + i % 3) for i in range(333)]
    p = Pool("bf16", "fp8", 4, 2, 64, 64, lens, seed=6)
    k, v = p.fill()
    news, total = [a for a, _ in lens], [b for _, b in lens]
    b, q = p.batch(news, total), p.normal(sum(news), 4, 64)
    for window, sinks in ((100, 4), (17, 65)):
        out = p.cache.attend_window(b, q, window, sinks)
        b.check()
        check_window(p, news, total, q, out, k, v, 0.125, window, sinks)


@pytest.mark.parametrize("kind", ["tokens", "drafts", "many"])
def test_a_captured_call_follows_the_lengths(kind):
    """Captured once, replayed at other lengths with eager work between the replays: the eager call's bits, from a workspace that keeps nothing; the answer in the queries' place."""
    news, heads, kv_heads = {"tokens": ([1, 1, 1], 8, 2), "drafts": ([6, 5, 1], 8, 2), "many": ([130, 70, 1], 64, 64)}[kind]
    longest = [4500, 700, 6000]
    p = Pool("bf16", "fp8", heads, kv_heads, 64, 64, list(zip(news, longest)), seed=13, max_len=6000)
    k, v = p.fill()
    b = p.batch(news, news)
    q = p.normal(sum(news), heads, 64)
    ws = torch.empty(max(p.cache.attend_window_workspace(b, 1700, 70), 256), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.cache.attend_window(b, q, 1700, 70, out=q, workspace=ws)
    for lens in (news, [200, 130, 64], longest, [1000, 700, 1], [4500, 200, 5999], longest):
        b.kv_len.copy_(torch.tensor(lens))
        rows = p.normal(sum(news), heads, 64)
        q.copy_(rows)
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        check_window(p, news, lens, rows, q, k, v, 0.125, 1700, 70)
        assert torch.equal(q, p.cache.attend_window(b, rows, 1700, 70))
    b.check()


def test_two_calls_at_once_on_streams_of_their_own():
    news, total = [5, 5], [5000, 3000]
    p = Pool("bf16", "fp8", 16, 2, 128, 64, list(zip(news, total)), seed=14)
    p.fill()
    batches = [asd.KVBatch(p.d_table[i:i + 1].contiguous(), torch.tensor([0, 5], dtype=torch.int32, device=DEV), torch.tensor([total[i]], dtype=torch.int32, device=DEV), 5, 5, p.cap)
               for i in range(2)]
    q = [p.normal(5, 16, 128) for _ in range(2)]
    want = [p.cache.attend_window(b, x, 2000, 4) for b, x in zip(batches, q)]
    out = [torch.empty_like(x) for x in q]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(8):
        for s, b, x, o in zip(streams, batches, q, out):
            with torch.cuda.stream(s):
                p.cache.attend_window(b, x, 2000, 4, out=o)
    torch.cuda.synchronize()
    for b, o, w in zip(batches, out, want):
        b.check()
        assert torch.equal(o, w)


def test_rows_in_front_of_the_first_position_are_zero():
    p = Pool("bf16", "fp8", 4, 2, 64, 64, [(5, 64), (3, 64), (2, 64)])
    p.fill()
    q = p.normal(10, 4, 64)
    b = p.batch([5, 3, 2], [2, 0, 64])
    out = p.cache.attend_window(b, q, 3, 1)
    assert bool((out[:3] == 0).all()) and bool((out[5:8] == 0).all()) and bool((out[3:5] != 0).any()) and bool((out[8:] != 0).any())
    with pytest.raises(asd.AsdError, match="rows or lengths"):
        b.check()


def test_positions_far_along_a_long_sequence():
    """Positions near 2^24 with a table whose entries behind the window are anything: the far end of what a batch may hold."""
    n, window, page = 2 ** 24, 300, 64
    args = (4, 2, 64, page, asd.DT_BF16, asd.DT_FP8)
    pages = torch.zeros(8 * asd.kv_page_bytes(*args), dtype=torch.uint8, device=DEV)
    cache = asd.KVCache(pages, *args)
    table = torch.full((1, n // page), -1, dtype=torch.int32, device=DEV)
    table[0, :1] = 7
    table[0, -7:] = torch.arange(7, dtype=torch.int32, device=DEV)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)      # noqa: E731
    g = torch.Generator(DEV).manual_seed(0)
    k, v = (torch.randn(400, 2, 64, generator=g, device=DEV).bfloat16() for _ in range(2))
    last = asd.KVBatch(table, i32([0, 400]), i32([n]), 400, 400, n)
    cache.append(last, None, k, v)
    k0, v0 = (torch.randn(64, 2, 64, generator=g, device=DEV).bfloat16() for _ in range(2))
    head = asd.KVBatch(table, i32([0, 64]), i32([64]), 64, 64, n)
    cache.append(head, None, k0, v0)
    (k, v), (k0, v0) = cache.read(last), cache.read(head)
    for rows in (1, 5, 90):
        b = asd.KVBatch(table, i32([0, rows]), i32([n]), rows, rows, n)
        q = torch.randn(rows, 4, 64, generator=g, device=DEV).bfloat16()
        out = cache.attend_window(b, q, window, 9)
        b.check()
        pos = torch.arange(9 + 400 - rows, 9 + 400, device=DEV)
        check("bf16", q, out, torch.cat([k0[:9], k]), torch.cat([v0[:9], v]), in_window(pos, 409, window, 9), 0.125, f"{rows} rows")


def test_refusals_of_the_binding():
    p = Pool("bf16", "fp8", 4, 2, 64, 64, [(2, 10)])
    p.fill()
    b, q = p.batch([2], [10]), p.normal(2, 4, 64)
    for window, sinks in ((0, 0), (-1, 4), (4, -1), (2 ** 31, 0), (1, 2 ** 40)):
        with pytest.raises(asd.AsdError):
            p.cache.attend_window(b, q, window, sinks)
    for bad in (q.float(), q[:1], q.cpu()):
        with pytest.raises(asd.AsdError):
            p.cache.attend_window(b, bad, 4)


@pytest.mark.parametrize("dtype,kv", COMBOS)
def test_a_long_conversation_in_a_few_pages(dtype, kv):
    """Prompt, drafts and tokens appended and attended to with a window, the pages behind it given to the tokens that come: five pages hold two conversations that would
    take sixteen."""
    h, heads, kv_heads, page, window, sinks = 64, 8, 2, 64, 70, 5
    args = (heads, kv_heads, h, page, asd.DT_BF16 if dtype == "bf16" else asd.DT_F32, {"f32": asd.DT_F32, "bf16": asd.DT_BF16, "fp8": asd.DT_FP8}[kv])
    cache = asd.KVCache(torch.full((10 * asd.kv_page_bytes(*args),), 0x7F, dtype=torch.uint8, device=DEV), *args)
    t = cache.torch_dtype
    gen = torch.Generator(DEV).manual_seed(3)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device=DEV).to(t)      # noqa: E731
    table = torch.full((2, 16), -1, dtype=torch.int32, device=DEV)
    rope = asd.rope_table(h, 1024)
    free, mine, lens, kept = [[0, 1, 2, 3, 4], [5, 6, 7, 8, 9]], [{}, {}], [0, 0], [([], []), ([], [])]
    for news in [[90, 33]] + [[5, 1], [1, 5]] * 30 + [[64, 100]] + [[1, 1]] * 40 + [[128, 100]]:
        for i in range(2):
            first = max(0, lens[i] - window + 1)        # the first key of the next row's window
            for j in [j for j in mine[i] if j and (j + 1) * page <= first]:
                free[i].append(mine[i].pop(j))
                table[i, j] = -1
            lens[i] += news[i]
            for j in range((lens[i] + page - 1) // page):
                if j not in mine[i] and (j + 1) * page > lens[i] - news[i]:
                    mine[i][j] = free[i].pop(0)
                    table[i, j] = mine[i][j]
        b = asd.KVBatch(table, torch.tensor([0, news[0], sum(news)], dtype=torch.int32, device=DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), sum(news), max(news), 1024)
        q = cache.append(b, normal(sum(news), heads, h), normal(sum(news), kv_heads, h), normal(sum(news), kv_heads, h), rope=rope, rot_dim=h)
        got = cache.read(b)
        out = cache.attend_window(b, q, window, sinks)
        b.check()
        at = 0
        for i, n in enumerate(news):
            for x, y in zip(kept[i], got):
                x.append(y[at:at + n])
            k, v = (torch.cat(x) for x in kept[i])
            pos = torch.arange(lens[i] - n, lens[i], device=DEV)
            check(dtype, q[at:at + n], out[at:at + n], k, v, in_window(pos, lens[i], window, sinks), h ** -0.5, f"conversation {i} at {lens[i]}")
            at += n
    assert min(lens) > 400 and max(len(x) for x in mine) <= 5


def test_an_engines_cache():
    """New rows attend to a window of what an engine's prompt pass has left in its pages."""
    import asd_inputs as si
    tiny = si.SHAPES["tiny"]
    eng = asd.Engine(asd.make_config(tiny, 256, page_tokens=64)).init_synthetic(0)
    eng.prefill(si.prompt(0, 200, tiny.vocab))
    k, v = (torch.from_numpy(x).cuda() for x in eng.get_kv(1, 0, 200))
    cache, table = eng.kv_cache(1)
    b = asd.KVBatch(table, torch.tensor([0, 3], dtype=torch.int32, device=DEV), torch.tensor([200], dtype=torch.int32, device=DEV), 3, 3, 256)
    q = torch.randn(3, tiny.n_heads, tiny.head_dim, generator=torch.Generator(DEV).manual_seed(1), device=DEV)
    out = cache.attend_window(b, q, 50, 4)
    b.check()
    pos = torch.arange(197, 200, device=DEV)
    check("f32", q, out, k.view(200, tiny.n_kv_heads, -1), v.view(200, tiny.n_kv_heads, -1), in_window(pos, 200, 50, 4), tiny.head_dim ** -0.5, "engine")
    eng.close()


@pytest.mark.parametrize("kv", ["fp8", "bf16"])
def test_many_first_tokens(kv):
    """First tokens of many chunks, whole ones among them, with values that are not finite in all of them, in front of windows of many rows and of few; a page of them missing."""
    news, total = [200, 3, 130], [3000, 2500, 2600]
    p = Pool("bf16", kv, 40, 40, 64, 64, list(zip(news, total)), seed=31)
    k, v = p.normal(sum(total), 40, 64), p.normal(sum(total), 40, 64)
    for i, key in enumerate(list(range(5, 1500, 97)) + [3000 + x for x in range(7, 1400, 111)] + [5500 + 640, 5500 + 700, 5500 + 1279]):
        v[key, i % 40, i % 64] = (math.nan, math.inf, -math.inf)[i % 3]
    whole = p.batch(total, total)
    p.cache.append(whole, None, k, v)
    k, v = (torch.split(x, total) for x in p.cache.read(whole))
    b, q = p.batch(news, total), p.normal(sum(news), 40, 64)
    for window, sinks in ((300, 1280), (500, 1300), (64, 1279)):
        out = p.cache.attend_window(b, q, window, sinks)
        b.check()
        check_window(p, news, total, q, out, k, v, 0.125, window, sinks)
    p.d_table[2, 7] = -1
    out = p.cache.attend_window(b, q, 300, 1280)
    with pytest.raises(asd.AsdError, match="pages"):
        b.check()
    seen = in_window(torch.arange(2470, 2600, device=DEV), 2600, 300, 1280)
    seen[:, 448:512] = False
    check("bf16", q[203:], out[203:], k[2], v[2], seen, 0.125, "a page of the first tokens is missing")
