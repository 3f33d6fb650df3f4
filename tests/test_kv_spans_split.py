"""How the attention with a window and the attention of shared beginnings cut a batch into work items, worked out on the CPU: whatever the arrays hold, a call has no more
items, and no more notes for the join, than its launch and its workspace have room for.  The cutting is written out from its description (asd_kv_spans.h,
asd_kv_plan.h) for fp32 rows and pages, whose tiles are of 16 rows; the sizes have to be the library's."""
import ctypes
import random

import pytest

import paper_2410_01028_amd as asd
from test_kv_split import UNITS, rows_of

H = 32


def up(x, n=256):
    return (x + n - 1) // n * n


def plan(form, heads, kv_heads, n_seqs, n_rows, max_new, chunks):
    """(most items, run's target, shortest run, cut, bytes of partial sums) of 16-row tiles."""
    group, seqs = heads // kv_heads, min(n_seqs, n_rows)
    whole = (n_rows * group // 16 + seqs) * kv_heads
    run, target = 16, 4 * UNITS
    if form in ("window", "both") and whole < UNITS:
        run, target = 4, UNITS
    if form == "front":
        rows = max_new * group
        run = min(8, max(4, (rows + 15) // 16 * seqs * kv_heads * chunks // UNITS))
    if form == "own":
        run, target = 2, 8 * UNITS
    most = (chunks + run // 2) // run
    cut = most > 1
    grid = min(whole + target, whole * most) if cut else whole
    return grid, target, run, cut, up(grid * 16 * H * 4), grid * 16 * 8


def notes(heads, kv_heads, n_seqs, n_rows):
    return up(64 + 48 * (n_rows * (heads // kv_heads) // 16 + min(n_seqs, n_rows)) * kv_heads)


def items(entries, group, kv_heads, target, shortest, cut):
    """entries: (rows, chunks).  (items, 16-row blocks of entries that are cut)."""
    tiles = [(n * group + 15) // 16 for n, _ in entries]
    run = max(shortest, sum(t * c for t, (_, c) in zip(tiles, entries)) * kv_heads // target + 1) if cut else 1 << 28
    splits = [max(1, (c + run // 2) // run) for _, c in entries]
    return sum(t * s for t, s in zip(tiles, splits)) * kv_heads, splits, tiles


def mended(row_start, lens, n_rows, max_new, cap):
    """(rows, position of the first, length) of every sequence."""
    out = []
    for (r0, n), f1, length in zip(rows_of(row_start, n_rows, max_new), row_start[1:], lens):
        first = length - f1 + r0
        n = max(0, min(n, cap - first))
        out.append((r0, n, first, min(max(first + n, 0), cap)))
    return out


def arrays(r):
    n_rows, n_seqs = r.randint(1, 200), r.randint(1, 150)
    max_new, cap = r.randint(1, n_rows), r.randint(64, 20000)
    start = [r.randint(-2, n_rows + 2) for _ in range(n_seqs + 1)]
    if r.random() < 0.5:
        start.sort()
    lens = [r.choice([r.randint(0, 100), cap, r.randint(0, cap), cap + 5, -3]) for _ in range(n_seqs)]
    heads, kv_heads = r.choice([(4, 4), (8, 2), (16, 1), (24, 8), (40, 40)])
    s = asd.KvShape(heads, kv_heads, H, 64, asd.DT_F32, asd.DT_F32)
    b = asd.KvBatch(1 << 20, 1 << 20, 1 << 20, 1 << 20, None, 4, (cap + 63) // 64, n_seqs, n_rows, max_new, cap)
    return start, lens, n_rows, n_seqs, max_new, cap, heads, kv_heads, s, b


def window_chunks(n, length, group, window, sinks):
    whole, sink = (length + 63) // 64, (sinks + 63) // 64
    if n * group <= 16:
        first = max(length - n - window + 1, 0) // 64
        return whole - first + sink if sink < first else whole
    tokens = min(n, (16 + group - 2) // group + 1 if 16 % group else 16 // group)
    return min(whole, sink + (window + tokens + 125) // 64)


def walked(n, length, group, window, sinks):
    """The most chunks that a tile of 16 rows walks, row by row."""
    most, base = 0, length - n
    for row in range(0, n * group, 16):
        first, last = base + row // group, base + (min(row + 16, n * group) - 1) // group
        keys = {c for p in (first, last) for c in range(max(p - window + 1, 0) // 64, p // 64 + 1)} | set(range(max(first - window + 1, 0) // 64, last // 64 + 1))
        most = max(most, len({c for c in keys | set(range((min(sinks, last + 1) + 63) // 64)) if 64 * c <= last}))
    return most


def test_chunks_of_a_window():
    r = random.Random(1)
    for _ in range(4000):
        n, group = r.randint(1, 90), r.choice([1, 2, 3, 4, 8, 16, 40])
        length = n + r.choice([0, r.randint(0, 200), r.randint(0, 3000)])
        window, sinks = min(r.choice([1, 5, 64, 100, 1000]), length), min(r.choice([0, 1, 64, 100, 700]), length)
        assert walked(n, length, group, window, sinks) <= window_chunks(n, length, group, window, sinks)


def test_any_arrays_fit_the_launch_of_a_window():
    r = random.Random(2)
    for _ in range(2500):
        start, lens, n_rows, n_seqs, max_new, cap, heads, kv_heads, s, b = arrays(r)
        group, window, sinks = heads // kv_heads, r.choice([1, 64, 500, 5000, 2 ** 31 - 1]), r.choice([0, 4, 300, 2 ** 31 - 1])
        size = asd._kv_lib().asd_kv_attend_window_workspace(ctypes.addressof(s), ctypes.addressof(b), window, sinks)
        window, sinks = min(window, cap), min(sinks, cap)
        tokens = min((16 + group - 2) // group + 1 if 16 % group else 16 // group, max_new)
        chunks = min((cap + 63) // 64, (sinks + 63) // 64 + (window + tokens + 125) // 64)
        grid, target, run, cut, o, ml = plan("window", heads, kv_heads, n_seqs, n_rows, max_new, chunks)
        blocks = notes(heads, kv_heads, n_seqs, n_rows)
        assert size == (blocks + o + ml if cut else 0)
        seqs = [(n, window_chunks(n, length, group, window, sinks)) for _, n, _, length in mended(start, lens, n_rows, max_new, cap)]
        assert all(c <= chunks for n, c in seqs if n)
        total, splits, tiles = items(seqs, group, kv_heads, target, run, cut)
        assert total <= grid
        assert 64 + 48 * kv_heads * sum(t for t, k in zip(tiles, splits) if k > 1) <= blocks


def groups_of(group_start, shared, start, lens, n_seqs, n_rows, cap):
    """(first sequence, end, tokens, first row, rows) of every group."""
    out, top, top_h = [], 0, 0
    clamp = lambda x, hi: min(max(x, 0), hi)        # noqa: E731
    for s0, s1, n in zip(group_start, group_start[1:], shared):
        good = s0 >= top and s1 >= s0 and s1 <= n_seqs
        top = max(top, clamp(s1, n_seqs))
        r0 = end = 0
        if good and s1 > s0:
            r0, end = clamp(start[s0], n_rows), clamp(start[s1], n_rows)
        rows = max(end - r0, 0) if r0 >= top_h else 0
        top_h = max(top_h, end)
        held = good and s1 > s0 and lens[s0] >= clamp(n, cap)
        out.append((s0 if good else 0, s1 if good else 0, clamp(n, cap) if held else 0, r0, rows))
    return out


@pytest.mark.parametrize("apart", [False, True])
def test_any_arrays_and_groups_fit_the_launch(apart):
    r, seen = random.Random(3), 0
    while seen < 1200:
        start, lens, n_rows, n_seqs, max_new, cap, heads, kv_heads, s, b = arrays(r)
        group, n_groups = heads // kv_heads, r.randint(1, min(n_seqs, 70))
        read = n_seqs * cap * kv_heads * H * 8
        if (n_seqs // 2 >= n_groups and n_rows * group <= 64 * n_seqs and ((cap >= 512 and read >= 40 << 20) or read >= 256 << 20)) != apart:
            continue
        seen += 1
        group_start = [r.randint(-2, n_seqs + 2) for _ in range(n_groups + 1)]
        if r.random() < 0.6:
            group_start.sort()
        shared = [r.choice([0, 64, r.randint(0, cap), cap + 1, -4, r.randint(0, 200)]) for _ in range(n_groups)]
        g = asd.KvGroups(1 << 20, 1 << 20, n_groups)
        size = asd._kv_lib().asd_kv_attend_shared_workspace(ctypes.addressof(s), ctypes.addressof(b), ctypes.addressof(g))
        seqs, blocks = mended(start, lens, n_rows, max_new, cap), notes(heads, kv_heads, n_seqs, n_rows)
        kinds = groups_of(group_start, shared, start, lens, n_seqs, n_rows, cap)
        claimed = [x for _, _, _, r0, n in kinds for x in range(r0, r0 + n)]
        assert len(claimed) == len(set(claimed)) and all(0 <= x < n_rows for x in claimed)
        low = [0] * n_seqs
        for i, (r0, n, first, length) in enumerate(seqs):
            for f0, f1, tokens, g0, rows in kinds:
                if f0 <= i < f1 and n and g0 <= r0 and r0 + n <= g0 + rows and length - n >= tokens:
                    low[i] = tokens
        chunks = (cap + 63) // 64
        if not apart:
            grid, target, run, cut, o, ml = plan("both", heads, kv_heads, n_seqs, n_rows, max_new, chunks + 1)
            assert size == (blocks + o + ml if cut else 0)
            total, splits, tiles = items([(n, (length + 63) // 64 + (x % 64 != 0)) for (_, n, _, length), x in zip(seqs, low)], group, kv_heads, target, run, cut)
            assert total <= grid and 64 + 48 * kv_heads * sum(t for t, k in zip(tiles, splits) if k > 1) <= blocks
            continue
        front, own = plan("front", heads, kv_heads, n_groups, n_rows, (n_rows + n_groups - 1) // n_groups, chunks), plan("own", heads, kv_heads, n_seqs, n_rows, max_new, chunks)
        assert size == blocks + up(front[4] + front[5]) + up(own[4] + own[5])
        total, _, _ = items([(rows, (tokens + 63) // 64) for _, _, tokens, _, rows in kinds if tokens], group, kv_heads, *front[1:4])
        assert total <= front[0]
        total, splits, tiles = items([(n, (length + 63) // 64 - x // 64) for (_, n, _, length), x in zip(seqs, low)], group, kv_heads, *own[1:4])
        assert total <= own[0] and 64 + 48 * kv_heads * sum(tiles) <= blocks      # (all rows are joined)


def test_the_last_round():
    """Tiles of 128 rows: those that fill whole rounds of two to a compute unit stay whole, the others fill one more at most, and have notes of all of their rows."""
    slots = 2 * UNITS
    s = asd.KvShape(8, 2, 64, 64, asd.DT_BF16, asd.DT_BF16)
    for n_rows, n_seqs in ((40000, 3), (4000, 3), (600, 600), (70, 2), (20000, 64)):
        b = asd.KvBatch(1 << 20, 1 << 20, 1 << 20, 1 << 20, None, 4, 1000, n_seqs, n_rows, n_rows, 60000)
        size = asd._kv_lib().asd_kv_attend_window_workspace(ctypes.addressof(s), ctypes.addressof(b), 5000, 4)
        whole = (n_rows * 4 // 128 + min(n_seqs, n_rows)) * 2
        sums = up(slots * 128 * 64 * 4) + slots * 128 * 8
        if not (whole * 8 > 4 * UNITS or size == 0 or size > sums):
            continue                                    # (few rows: 16 to a tile)
        most = 5000 // 64 // 8
        for total in range(1, whole + 1):
            rest = total % slots
            k = max(1, min(slots // rest, most)) if rest else 1
            assert (rest * k if k > 1 else 0) <= slots
            if k > 1:
                assert size >= up(64 + 48 * rest * 8) + sums
