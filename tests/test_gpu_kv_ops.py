"""The operators over a paged cache of several sequences (KVCache.append, attend, read; rope_table) against 64 bits.

Tolerances, fixed before the first run.  Rounding to a type is off by at most half a step (bf16 2^-8, fp32 2^-24 of the value).
append: the norm and the rotation are a sum of h squares and at most five products and sums per value: (h + 16) 2^-24 of the largest
magnitudes that enter a value (|a| + |b| of its pair), then one rounding.
attend: a score is a sum of h products, off by E = h 2^-24 scale sum|q||k| at most; weights are off by 2E from the scores of both sides of
the softmax and 2^-20 from the exponentials (an argument of up to 2^3 that counts, in steps of 2^-24, and an ulp of the function), bf16 rows round each
by 2^-8 more; sums over n keys add n 2^-24; all of it times sum p|v|; then one rounding.
"""
import math

import pytest
import torch

import paper_2410_01028_amd as asd
from kv_reference import attention, exponent, held, place, prepared

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": (torch.float32, asd.DT_F32), "bf16": (torch.bfloat16, asd.DT_BF16), "fp8": (None, asd.DT_FP8)}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
COMBOS = [("bf16", "fp8"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "fp8")]


class Pool:
    """A cache whose pages start as `fill` bytes, and batches of sequences over it."""

    def __init__(self, dtype, kv, heads, kv_heads, h, page, lens, seed=0, fill=0x7F, max_len=None, spare=2):
        self.t, self.dtype, self.kv, self.h, self.heads, self.kv_heads, self.page = TYPES[dtype][0], dtype, kv, h, heads, kv_heads, page
        self.lens = lens
        self.each = max(1, max((b + page - 1) // page for _, b in lens))
        n = len(lens) * self.each + spare
        g = torch.Generator().manual_seed(seed)
        self.table = torch.randperm(n, generator=g)[:len(lens) * self.each].view(len(lens), self.each).int()
        args = (heads, kv_heads, h, page, TYPES[dtype][1], TYPES[kv][1])
        self.pages = torch.full((n, asd.kv_page_bytes(*args)), fill, dtype=torch.uint8, device=DEV)
        self.cache = asd.KVCache(self.pages, *args)
        self.gen = torch.Generator(DEV).manual_seed(seed)
        self.cap = max_len or self.each * page
        self.d_table = self.table.to(DEV)

    def batch(self, news, lens, extra=0, max_new=None):
        start = [0]
        for n in news:
            start.append(start[-1] + n)
        return asd.KVBatch(self.d_table, torch.tensor(start, dtype=torch.int32, device=DEV), torch.tensor(lens, dtype=torch.int32, device=DEV),
                           n_rows=start[-1] + extra, max_new=max_new or max(1, max(news)), max_len=self.cap)

    def normal(self, *shape, scale=1.0):
        return (torch.randn(*shape, generator=self.gen, device=DEV) * scale).to(self.t)

    def fill(self):
        """Whole sequences of random rows into the pages; their values as the cache holds them."""
        news = [b for _, b in self.lens]
        rows = sum(news)
        k, v = self.normal(rows, self.kv_heads, self.h), self.normal(rows, self.kv_heads, self.h)
        whole = self.batch(news, news)
        self.cache.append(whole, None, k, v)
        k, v = self.cache.read(whole)
        whole.check()
        return torch.split(k, news), torch.split(v, news)


def close(got, want, tol, what):
    got = got.double()
    assert torch.equal(got.isnan(), want.isnan()), what
    ok = want.isfinite()
    assert torch.equal(got[~ok & ~want.isnan()], want[~ok & ~want.isnan()]), what
    d = torch.where(ok, (got - want).abs() - tol, torch.zeros_like(tol))
    assert float(d.max()) <= 0, f"{what}: {float(d.max())} over the tolerance, difference {float((got - want)[ok].abs().max())}"


LENS = [(1, 1), (3, 3), (0, 9), (16, 80), (17, 64), (5, 131), (70, 70), (1, 200), (33, 97)]


@pytest.mark.parametrize("dtype,kv", COMBOS)
@pytest.mark.parametrize("h,heads,kv_heads,rot,inter,norm", [(128, 8, 2, 128, False, True), (128, 3, 3, 64, True, False), (64, 10, 5, 48, False, False),
                                                             (64, 4, 4, 64, True, True), (32, 6, 2, 16, False, True), (32, 1, 1, 0, False, False)])
def test_append_and_read(dtype, kv, h, heads, kv_heads, rot, inter, norm):
    p = Pool(dtype, kv, heads, kv_heads, h, 64, LENS, seed=h + rot)
    news, lens = [a for a, _ in LENS], [b for _, b in LENS]
    before_news = [b - a for a, b in LENS]
    old = p.normal(2, sum(before_news), kv_heads, h)
    before = p.batch(before_news, before_news)
    p.cache.append(before, None, old[0], old[1])
    old_k, old_v = p.cache.read(before)
    rows, extra = sum(news), 3
    # slices of one buffer of fused rows, as a QKV product leaves them
    fused = p.normal(rows + extra, heads + 2 * kv_heads, h, scale=3.0)
    q, k, v = fused[:, :heads], fused[:, heads:heads + kv_heads], fused[:, heads + kv_heads:]
    k[1] *= 1e-3
    gains = [(1 + 0.2 * torch.randn(h, device=DEV)) if norm else None for _ in range(2)]
    positions = torch.cat([torch.arange(b - a, b) for a, b in LENS])
    table = asd.rope_table(rot, max(lens), theta=500.0) if rot else None
    out = torch.full((rows + extra, heads, h), 7.0, dtype=p.t, device=DEV)
    batch = p.batch(news, lens, extra=extra)
    p.cache.append(batch, q, k, v, q_out=out, rope=table, rot_dim=rot, interleaved=inter, q_gain=gains[0], k_gain=gains[1], eps=1e-5)
    got_k, got_v = p.cache.read(batch, *(torch.full((rows + extra, kv_heads, h), 7.0, dtype=p.t, device=DEV) for _ in range(2)))
    batch.check()
    for t in (out, got_k, got_v):
        assert bool((t[rows:] == 7.0).all())            # rows behind the last sequence: as they were
    cs = table[positions.to(DEV)] if rot else None
    e = (h + 16) * 2.0 ** -24
    for got, x, gain, name in ((out, q, gains[0], "q"), (got_k, k, gains[1], "k"), (got_v, v, None, "v")):
        turn = cs if name != "v" else None
        want = prepared(x[:rows], gain, 1e-5, turn, rot if name != "v" else 0, inter)
        size = prepared(x[:rows], gain, 1e-5, None, 0, False).abs()
        if turn is not None and rot:                    # the other of the pair: what a quarter turn brings in its place
            quarter = torch.tensor([0.0, 1.0], device=DEV).expand_as(turn)
            size = size + torch.cat([prepared(size, None, 0, quarter, rot, inter).abs()[..., :rot], torch.zeros_like(size[..., rot:])], -1)
        slack = e * size
        if gain is None:
            slack[..., rot if name != "v" else 0:] = 0.0        # passed through: exactly its rounding
        if name == "q" or kv != "fp8":
            close(got[:rows], want, slack + (want.abs() + slack) * HALF[dtype], name)
        else:
            value, border, step = held(want)
            near = border < slack                       # a step further where the value lies on a border
            close(got[:rows], value, torch.where(near, step * 1.001, torch.zeros_like(step)), name)
            assert float(near.double().mean()) < 0.01
    again_k, again_v = p.cache.read(before)              # what was there before
    before.check()
    assert torch.equal(again_k, old_k) and torch.equal(again_v, old_v)


@pytest.mark.parametrize("kv,h", [("fp8", 128), ("fp8", 64), ("fp8", 32), ("bf16", 128), ("f32", 64)])
def test_pages_have_the_documented_layout(kv, h):
    dtype = "f32" if kv == "f32" else "bf16"
    p = Pool(dtype, kv, 2, 2, h, 128, [(0, 128)], fill=0)
    k, v = p.fill()
    size = {"f32": 4, "bf16": 2, "fp8": 1}[kv]
    chunk = 2 * 64 * h * size + (128 if kv == "fp8" else 0)
    page = p.pages[int(p.table[0, 0])].cpu().view(2, 2, chunk)
    view = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}[kv]
    for head, pos, dim in [(0, 0, 0), (1, 127, h - 1), (0, 37, 5), (1, 64, h // 2 + 3), (0, 91, 17), (1, 18, 30)]:
        raw = page[head, pos // 64]
        for i, t in enumerate((k[0], v[0])):
            at = place(kv, h, pos % 64, dim)[i]
            x = float(raw[at:at + size].clone().view(view).float())
            if kv == "fp8":
                x *= 2.0 ** (int(raw[2 * 64 * h + 64 * i + pos % 64]) - 127)
            assert x == float(t[pos, head, dim])


def test_eight_bits_extremes():
    """Rows of zeros, of one value, tiny and huge ones, and ones with NaN and infinities: the scale comes from the finite values."""
    p = Pool("f32", "fp8", 1, 1, 64, 64, [(8, 8)])
    x = torch.randn(8, 1, 64, generator=torch.Generator().manual_seed(3))
    x[0], x[1] = 0.0, 448.0
    x[2], x[3] = x[2] * 1e-36, x[3] * 1e37
    x[4, 0, :3] = torch.tensor([math.nan, math.inf, -math.inf])
    x[5] = math.inf
    x[6, 0, 0], x[7] = 448.0001, 1.75 * 2.0 ** -30
    x = x.to(DEV)
    b = p.batch([8], [8])
    p.cache.append(b, None, x, x)
    for got in p.cache.read(b):
        want, _, _ = held(x.double())
        assert torch.equal(torch.nan_to_num(got, 123.0), torch.nan_to_num(want.float(), 123.0))
        assert float((got[6] - x[6]).abs()[0, 0]) <= 32 and float(got[7, 0, 0]) == 1.75 * 2.0 ** -30
    assert float(exponent(x.double())[6]) == 1.0


ATTEND = {
    "tokens": [(1, 1), (1, 63), (1, 64), (1, 65), (0, 7), (1, 257), (1, 1000), (1, 2500)],
    "drafts": [(5, 5), (3, 70), (5, 600), (1, 129), (4, 64)],
    "chunks": [(64, 64), (70, 333), (1, 20), (130, 1200)],
    "one": [(1, 700)],
}


def check_attend(p, news, lens, q, out, k, v, scale):
    at = 0
    for i, (n, length) in enumerate(zip(news, lens)):
        if n:
            want, size, big = attention(q[at:at + n], k[i][:length], v[i][:length], length - n, scale)
            e = 2 * p.h * 2.0 ** -24 * big[..., None] + 2.0 ** -20 + length * 2.0 ** -24 + (2.0 ** -8 if p.dtype == "bf16" else 0.0)
            close(out[at:at + n], want, size * e + (want.abs().nan_to_num(0, 0, 0) + size * e) * HALF[p.dtype], f"sequence {i}")
        at += n


@pytest.mark.parametrize("dtype,kv", COMBOS)
@pytest.mark.parametrize("lens", list(ATTEND))
@pytest.mark.parametrize("h,heads,kv_heads,page", [(128, 8, 1, 64), (128, 4, 4, 192), (64, 15, 5, 64), (32, 6, 2, 128)])
def test_attend(dtype, kv, lens, h, heads, kv_heads, page):
    p = Pool(dtype, kv, heads, kv_heads, h, page, ATTEND[lens], seed=h)
    k, v = p.fill()
    news, total = [a for a, _ in ATTEND[lens]], [b for _, b in ATTEND[lens]]
    rows = sum(news)
    wide = p.normal(rows + 2, heads + 3, h, scale=2.0)
    q = wide[:, 1:heads + 1]
    out = torch.full((rows + 2, heads, h), 7.0, dtype=p.t, device=DEV)
    b = p.batch(news, total, extra=2)
    p.cache.attend(b, q, out=out)
    b.check()
    assert bool((out[rows:] == 7.0).all())
    check_attend(p, news, total, q, out, k, v, h ** -0.5)


@pytest.mark.parametrize("dtype,kv", COMBOS)
@pytest.mark.parametrize("news,kv_heads", [((40, 6, 90), 64), ((40, 6, 90), 2), ((5, 3, 4), 2), ((1, 6, 1), 2)], ids=["many rows", "chunks", "drafts", "tokens"])
@pytest.mark.parametrize("h", [64, 128])
def test_values_that_are_not_finite_stay_where_they_are_seen(dtype, kv, news, kv_heads, h):
    """Infinities and NaN in V and NaN in K at keys that some rows of the call do not see, and in chunks that all rows see."""
    total = [100, 6, 130]
    p = Pool(dtype, kv, 2 * kv_heads, kv_heads, h, 64, list(zip(news, total)), seed=1)
    k, v = p.normal(sum(total), kv_heads, h), p.normal(sum(total), kv_heads, h)
    v[70, 0, 3], v[95, 0, 7], v[95, 1, 9], v[97, 0, 7], v[103, 1, 60], v[220, 0, 33] = math.inf, math.inf, math.nan, -math.inf, -math.inf, math.nan
    v[110, 1, 2], v[233, 1, 5] = math.inf, -math.inf
    k[104, 0, 5] = math.nan
    whole = p.batch(total, total)
    p.cache.append(whole, None, k, v)
    k, v = (torch.split(x, total) for x in p.cache.read(whole))
    b = p.batch(news, total)
    q = p.normal(sum(news), 2 * kv_heads, h)
    out = p.cache.attend(b, q)
    b.check()
    one, two = news[0], news[0] + news[1]
    assert bool(out[two - 2:two, :2].isnan().all()) and bool(out[two - 2:two, 2:, :60].isfinite().all())      # the K of key 4, its own KV head
    check_attend(p, [one], total[:1], q[:one], out[:one], k[:1], v[:1], h ** -0.5)
    check_attend(p, [news[2]], total[2:], q[two:], out[two:], k[2:], v[2:], h ** -0.5)


@pytest.mark.parametrize("kv", ["fp8", "bf16"])
@pytest.mark.parametrize("h,heads,kv_heads,page", [(128, 40, 40, 64), (128, 64, 8, 192), (64, 64, 8, 64), (64, 40, 40, 128)])
def test_attend_many_rows(kv, h, heads, kv_heads, page):
    """Batches whose tiles fill the card: 128 rows share a chunk (prompts, chunks behind a context, a single token and nothing among them)."""
    news, total = [64, 70, 1, 130, 0, 200, 17, 2], [64, 333, 20, 1200, 9, 200, 17, 2]
    p = Pool("bf16", kv, heads, kv_heads, h, page, list(zip(news, total)), seed=h)
    k, v = p.fill()
    q = p.normal(sum(news) + 3, heads + 2, h, scale=2.0)[:, 1:heads + 1]
    out = torch.full((sum(news) + 3, heads, h), 7.0, dtype=p.t, device=DEV)
    b = p.batch(news, total, extra=3)
    p.cache.attend(b, q, out=out)
    b.check()
    assert bool((out[sum(news):] == 7.0).all())
    check_attend(p, news, total, q, out, k, v, h ** -0.5)
    p.d_table[3, 1] = -1                                 # a page that is not there, in the middle of the fourth sequence
    p.cache.attend(b, q, out=out)
    with pytest.raises(asd.AsdError, match="pages"):
        b.check()
    keep = torch.cat([torch.arange(page), torch.arange(2 * page, 1200)]).to(DEV)
    at = 64 + 70 + 1
    want, size, big = attention(q[at:at + 130], k[3][keep], v[3][keep], 1200 - page - 130, h ** -0.5)
    e = 2 * h * 2.0 ** -24 * big[..., None] + 2.0 ** -20 + 1200 * 2.0 ** -24 + 2.0 ** -8
    close(out[at:at + 130], want, size * e + (want.abs() + size * e) * 2.0 ** -8, "hidden page")


def test_attend_many_rows_over_many_pages():
    """Runs of more pages than a wave holds at a time."""
    news, total = [1024, 1000], [4400, 4300]
    p = Pool("bf16", "fp8", 64, 64, 64, 64, list(zip(news, total)), seed=8)
    k, v = p.fill()
    q = p.normal(2024, 64, 64)
    b = p.batch(news, total)
    out = p.cache.attend(b, q)
    b.check()
    check_attend(p, news, total, q, out, k, v, 0.125)


@pytest.mark.parametrize("kv", ["fp8", "bf16"])
def test_long_and_lopsided_batches(kv):
    """One long sequence among short ones: its keys are cut into runs and joined, for a token, a few rows and chunks of many."""
    for news, total in (((1, 1, 1, 1), (20000, 40, 1, 700)), ((6, 0, 2, 6), (9000, 40, 2, 7000)), ((150, 1, 90, 3), (6000, 40, 90, 2100)), ((300, 1, 90, 3), (9000, 40, 90, 2100))):
        p = Pool("bf16", kv, 8, 2, 128, 256, list(zip(news, total)), seed=3)
        k, v = p.fill()
        b = p.batch(news, total)
        q = p.normal(sum(news), 8, 128, scale=2.0)
        out = p.cache.attend(b, q)
        b.check()
        check_attend(p, news, total, q, out, k, v, 128 ** -0.5)


def test_many_sequences():
    """More sequences than a wave looks at at a time, some without new rows."""
    lens = [(i % 3, 1 + (i * 37) % 150 + i % 3) for i in range(333)]
    p = Pool("bf16", "fp8", 4, 2, 64, 64, lens, seed=6)
    k, v = p.fill()
    news, total = [a for a, _ in lens], [b for _, b in lens]
    b = p.batch(news, total)
    q, kn, vn = p.normal(sum(news), 4, 64), p.normal(sum(news), 2, 64), p.normal(sum(news), 2, 64)
    turned = p.cache.append(b, q, kn, vn)
    assert torch.equal(turned, q)
    whole = p.batch(total, total)
    k, v = (torch.split(x, total) for x in p.cache.read(whole))
    out = p.cache.attend(b, q)
    b.check(), whole.check()
    check_attend(p, news, total, q, out, k, v, 0.125)


def test_pages_far_apart():
    """Offsets past 2^32 bytes: a pool of more than 8 GiB, the sequence's pages at its ends."""
    args = (8, 8, 128, 256, asd.DT_BF16, asd.DT_BF16)
    each = asd.kv_page_bytes(*args)
    n = 9 * 2 ** 30 // each
    pages = torch.empty(n * each, dtype=torch.uint8, device=DEV)
    cache = asd.KVCache(pages, *args)
    g = torch.Generator(DEV).manual_seed(0)
    k, v, q = (torch.randn(600, 8, 128, generator=g, device=DEV).bfloat16() for _ in range(3))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)      # noqa: E731
    whole = asd.KVBatch(i32([[n - 1, 0, n - 2]]), i32([0, 600]), i32([600]), 600, 600, 600)
    turned = cache.append(whole, q, k, v)
    rk, rv = cache.read(whole)
    assert torch.equal(turned, q) and torch.equal(rk, k) and torch.equal(rv, v)
    out = cache.attend(whole, q)
    few = asd.KVBatch(whole.page_table, i32([0, 2]), whole.kv_len, 2, 2, 600)
    out2 = cache.attend(few, q[598:])
    whole.check(), few.check()
    want, size, big = attention(q, k, v, 0, 128 ** -0.5)
    e = 2 * 128 * 2.0 ** -24 * big[..., None] + 2.0 ** -20 + 600 * 2.0 ** -24 + 2.0 ** -8
    close(out, want, size * e + (want.abs() + size * e) * 2.0 ** -8, "rows")
    close(out2, want[598:], (size * e + (want.abs() + size * e) * 2.0 ** -8)[598:], "few")


def test_in_place_and_aligned_slices():
    """Queries prepared in place; rows with strides; pages that are a slice of a larger buffer."""
    args = (4, 2, 64, 64, asd.DT_BF16, asd.DT_FP8)
    each = asd.kv_page_bytes(*args)
    buffer = torch.zeros(16 + 3 * each, dtype=torch.uint8, device=DEV)
    cache = asd.KVCache(buffer[16:], *args)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)      # noqa: E731
    b = asd.KVBatch(i32([[2, 0]]), i32([0, 70]), i32([70]), 70, 70, 128)
    fused = torch.randn(70, 10, 64, device=DEV).bfloat16()
    q, k, v = fused[:, :4], fused[:, 4:6], fused[:, 6:8]
    table, gain = asd.rope_table(64, 70), torch.full((64,), 1.5, device=DEV)
    apart = cache.append(b, q.clone(), k, v, rope=table, rot_dim=64, q_gain=gain)
    rest = fused[:, 4:].clone()
    assert cache.append(b, q, k, v, q_out=q, rope=table, rot_dim=64, q_gain=gain) is q
    assert torch.equal(q, apart) and torch.equal(fused[:, 4:], rest) and bool((buffer[:16] == 0).all())
    b.check()


def test_refusals_of_the_binding():
    p = Pool("bf16", "fp8", 4, 2, 64, 64, [(2, 10)])
    p.fill()
    b = p.batch([2], [10])
    q, k = p.normal(2, 4, 64), p.normal(2, 2, 64)
    for bad in (q.float(), q[:1], q[:, :3], q.transpose(0, 1), q.cpu(), p.normal(2, 4, 128)[..., ::2], p.normal(2, 8, 64)[:, ::2]):
        with pytest.raises(asd.AsdError):
            p.cache.attend(b, bad)
    with pytest.raises(asd.AsdError):
        p.cache.attend(b, q, workspace=torch.empty(4, dtype=torch.uint8))
    with pytest.raises(asd.AsdError):
        p.cache.append(b, None, k, k, q_out=q)
    for kw in (dict(rope=torch.zeros(10, 32, 2, device=DEV).double(), rot_dim=64), dict(rope=torch.zeros(10, 16, 2, device=DEV), rot_dim=64), dict(rot_dim=64),
               dict(q_gain=torch.ones(32, device=DEV)), dict(k_gain=torch.ones(64))):
        with pytest.raises(asd.AsdError):
            p.cache.append(b, q, k, k, **kw)
    for bad in ((p.d_table.long(), b.row_start, b.kv_len), (p.d_table, b.row_start[:1], b.kv_len), (p.d_table, b.row_start, b.kv_len.cpu()), (p.table, b.row_start.cpu(), b.kv_len.cpu())):
        with pytest.raises(asd.AsdError):
            asd.KVBatch(*bad, n_rows=2, max_new=2, max_len=10)
    with pytest.raises(asd.AsdError):
        asd.KVCache(p.pages.view(-1)[:-1], 4, 2, 64, 64)


def test_rows_without_keys_are_zero():
    """kv_len below the number of new rows: the rows in front have no position; an empty sequence has no keys at all."""
    p = Pool("bf16", "fp8", 4, 2, 64, 64, [(5, 64), (3, 64), (2, 64)])
    p.fill()
    q = p.normal(10, 4, 64)
    b = p.batch([5, 3, 2], [2, 0, 64])
    out = p.cache.attend(b, q)
    assert bool((out[:3] == 0).all()) and bool((out[5:8] == 0).all()) and bool((out[3:5] != 0).any()) and bool((out[8:] != 0).any())
    with pytest.raises(asd.AsdError, match="rows or lengths"):
        b.check()
    b.check()                                            # reported once


def test_large_scores_and_scale():
    """Scores of thousands: the running maximum keeps the sums finite."""
    p = Pool("f32", "f32", 2, 1, 64, 64, [(3, 300)])
    k, v = p.fill()
    q = p.normal(3, 2, 64, scale=50.0)
    b = p.batch([3], [300])
    out = p.cache.attend(b, q, scale=3.0)
    assert bool(out.isfinite().all())
    check_attend(p, [3], [300], q, out, k, v, 3.0)


def test_pages_out_of_range_are_hidden_and_reported():
    p = Pool("bf16", "bf16", 2, 1, 64, 64, [(1, 256), (1, 256)])
    k, v = p.fill()
    for bad in (-1, p.cache.n_pages, 2 ** 31 - 1):
        p.d_table.copy_(p.table)
        p.d_table[0, 1] = bad
        q = p.normal(2, 2, 64)
        b = p.batch([1, 1], [256, 256])
        out = p.cache.attend(b, q)
        keep = torch.cat([torch.arange(64), torch.arange(128, 256)]).to(DEV)
        want, size, _ = attention(q[:1], k[0][keep], v[0][keep], 191, 0.125)
        close(out[:1], want, size * 0.01 + want.abs() * 2.0 ** -8, "hidden page")
        check_attend(p, [1], [256], q[1:], out[1:], k[1:], v[1:], 0.125)
        with pytest.raises(asd.AsdError, match="pages"):
            b.check()
        whole = p.batch([256, 256], [256, 256])
        rk, _ = p.cache.read(whole, *(torch.full((512, 1, 64), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)))
        assert bool((rk[64:128] == 7.0).all()) and torch.equal(rk[256:], k[1])
        with pytest.raises(asd.AsdError, match="pages"):
            whole.check()
        saved = p.pages.clone()
        p.cache.append(p.batch([1, 0], [100, 256]), None, p.normal(1, 1, 64), p.normal(1, 1, 64))
        assert torch.equal(saved, p.pages)               # nothing was written


def test_arrays_out_of_range_are_cut_and_reported():
    p = Pool("bf16", "fp8", 2, 1, 64, 64, [(4, 128), (4, 128)])
    p.fill()
    q = p.normal(8, 2, 64)
    for start, lens in (([0, -5, 8], [128, 128]), ([0, 4, 2 ** 31 - 1], [128, 128]), ([-2 ** 31, 4, 8], [128, 128]), ([0, 4, 8], [2 ** 31 - 1, -3]), ([0, 4, 8], [129, 128])):
        b = asd.KVBatch(p.d_table, torch.tensor(start, dtype=torch.int32, device=DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), 8, 4, 128)
        out = p.cache.attend(b, q, out=torch.zeros_like(q))      # (rows that no sequence has stay as they are)
        assert bool(out.isfinite().all())
        with pytest.raises(asd.AsdError, match="rows or lengths"):
            b.check()
    table = asd.rope_table(64, 100)
    b = p.batch([4, 0], [128, 128])
    p.cache.append(b, q[:4], q[:4, :1], q[:4, :1], rope=table, rot_dim=64)
    with pytest.raises(asd.AsdError, match="rotary"):
        b.check()


def test_runs_together_as_a_serving_loop_and_in_a_graph():
    """Prompts in, then tokens one by one: append, attend, lengths updated on the device; the same step captured once and replayed."""
    lens0, steps, heads, kv_heads, h = [37, 64, 5, 130], 6, 8, 2, 64
    rows = []
    for captured in (False, True):
        p = Pool("bf16", "fp8", heads, kv_heads, h, 64, [(1, n + steps) for n in lens0], seed=4)
        table = asd.rope_table(h, 256)
        prompt = p.batch(lens0, lens0)
        q, k, v = p.normal(sum(lens0), heads, h), p.normal(sum(lens0), kv_heads, h), p.normal(sum(lens0), kv_heads, h)
        rows.append([p.cache.attend(prompt, p.cache.append(prompt, q, k, v, rope=table, rot_dim=h))])
        prompt.check()
        b = p.batch([1] * 4, lens0)
        x = [p.normal(steps, 4, n, h) for n in (heads, kv_heads, kv_heads)]
        q, k, v = (t[0].clone() for t in x)
        turned, out = torch.empty_like(q), torch.empty_like(q)
        ws = torch.empty(p.cache.attend_workspace(b), dtype=torch.uint8, device=DEV)

        def step():
            b.kv_len.add_(1)
            p.cache.append(b, q, k, v, q_out=turned, rope=table, rot_dim=h)
            p.cache.attend(b, turned, out=out, workspace=ws)

        if captured:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        for i in range(steps):
            for t, s in zip((q, k, v), x):
                t.copy_(s[i])
            graph.replay() if captured else step()
            rows[-1].append(out.clone())
            ws.fill_(0xFF)                               # the workspace keeps nothing from call to call
        b.check()
        whole = p.batch([n + steps for n in lens0], [n + steps for n in lens0])
        kk, vv = p.cache.read(whole)
        sizes = [n + steps for n in lens0]
        check_attend(p, [1] * 4, sizes, turned, out, torch.split(kk, sizes), torch.split(vv, sizes), h ** -0.5)
    assert all(torch.equal(a, b) for a, b in zip(*rows))


def test_on_another_stream_and_repeated():
    """The same call twice and on a stream of its own: the same bits."""
    p = Pool("bf16", "fp8", 8, 2, 128, 64, [(1, 3000), (1, 90)], seed=2)
    p.fill()
    q = p.normal(2, 8, 128)
    b = p.batch([1, 1], [3000, 90])
    a = p.cache.attend(b, q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = p.cache.attend(b, q)
    side.synchronize()
    assert torch.equal(a, p.cache.attend(b, q)) and torch.equal(a, c)


@pytest.mark.parametrize("kind,kw", [(asd.ROPE_PLAIN, {}), (asd.ROPE_LINEAR, dict(factor=4.0)), (asd.ROPE_BANDS, dict(factor=8.0, low=1.0, high=4.0, trained=512.0)),
                                     (asd.ROPE_RAMP, dict(factor=4.0, low=1.0, high=32.0, trained=2048.0, gain=1.1386))])
def test_rope_table(kind, kw):
    rot, n, theta = 64, 3001, 10000.0
    got = asd.rope_table(rot, n, theta=theta, kind=kind, **kw).cpu().double()
    f = [theta ** (-2 * j / rot) for j in range(rot // 2)]
    if kind:
        fac, tr = kw["factor"], kw.get("trained")
        if kind == asd.ROPE_LINEAR:
            f = [x / fac for x in f]
        elif kind == asd.ROPE_BANDS:
            keep = [min(1.0, max(0.0, (tr * x / (2 * math.pi) - kw["low"]) / (kw["high"] - kw["low"]))) for x in f]
            f = [k * x + (1 - k) * x / fac for k, x in zip(keep, f)]
        else:
            at = [rot * math.log(tr / (2 * math.pi * t)) / (2 * math.log(theta)) for t in (kw["high"], kw["low"])]
            lo, hi = math.floor(at[0]), math.ceil(at[1])
            keep = [1 - min(1.0, max(0.0, (j - lo) / (hi - lo))) for j in range(rot // 2)]
            f = [k * x + (1 - k) * x / fac for k, x in zip(keep, f)]
    a = torch.arange(n, dtype=torch.float64)[:, None] * torch.tensor(f, dtype=torch.float64)
    want = torch.stack([a.cos(), a.sin()], -1) * kw.get("gain", 1.0)
    assert float((got - want).abs().max()) <= 2.0 ** -24 * 1.2 + 1e-11
