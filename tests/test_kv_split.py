"""How asd_kv_attend cuts a batch into work items, worked out on the CPU: whatever row_start and kv_len hold, the items of a batch are no more than the
workspace that asd_kv_attend_workspace asks for has room for.  The library gives the room; the cutting is written out here from its description
(asd.h: which rows a sequence has; asd_kv.h: tiles, runs, splits)."""
import ctypes
import random

import pytest

import paper_2410_01028_amd as asd

UNITS = 256        # compute units: what the library takes where it finds no device


def room(heads, kv_heads, h, kv, nt, n_seqs, n_rows, max_new, max_len):
    """Work items that the workspace has room for; nt: 16-row blocks of a tile of the kernel that such a batch takes (0: nothing is cut)."""
    s = asd.KvShape(heads, kv_heads, h, 64, asd.DT_BF16, kv)
    b = asd.KvBatch(1 << 20, 1 << 20, 1 << 20, 1 << 20, None, 4, (max_len + 63) // 64, n_seqs, n_rows, max_new, max_len)
    size = asd._kv_lib().asd_kv_attend_workspace(ctypes.addressof(s), ctypes.addressof(b))
    return size // (16 * nt * (4 * h + 8))


def rows_of(row_start, n_rows, max_new, disjoint=True):
    """(first row, rows) of every sequence; a sequence that begins in front of the end of an earlier one has none."""
    out, top = [], 0
    for f0, f1 in zip(row_start, row_start[1:]):
        r0 = min(max(f0, 0), n_rows)
        end = min(max(f1, r0), n_rows)
        out.append((r0, 0 if disjoint and r0 < top else min(end - r0, max_new)))
        top = max(top, end)
    return out


def items(rows, lens, group, kv_heads, nt, cap):
    tiles = [(n * group + 16 * nt - 1) // (16 * nt) for _, n in rows]
    chunks = [(min(max(x, 0), cap) + 63) // 64 for x in lens]
    run = max(16, sum(t * c for t, c in zip(tiles, chunks)) * kv_heads // (4 * UNITS) + 1)
    return sum(t * max(1, (c + run // 2) // run) * kv_heads for t, c in zip(tiles, chunks))


OVERLAP = [     # heads, KV heads, dim, cache type, 16-row blocks, sequences, rows, max_len, lengths: row_start 0, N, 0, N, ..
    (64, 8, 128, asd.DT_FP8, 8, 128, 64, 8192, [64] * 126 + [8192, 64]),
    (128, 16, 128, asd.DT_BF16, 8, 5, 100, 1536, [1536] * 5),
    (32, 32, 64, asd.DT_FP8, 1, 40, 9, 3000, [3000] * 40)]


@pytest.mark.parametrize("case", OVERLAP, ids=["one long sequence", "five of a length", "tiles of 16 rows"])
def test_rows_that_several_sequences_claim(case):
    heads, kv_heads, h, kv, nt, n_seqs, n_rows, max_len, lens = case
    start = [n_rows * (i % 2) for i in range(n_seqs + 1)]
    have = room(heads, kv_heads, h, kv, nt, n_seqs, n_rows, n_rows, max_len)
    each = heads // kv_heads
    assert 0 < items(rows_of(start, n_rows, n_rows), lens, each, kv_heads, nt, max_len) <= have
    assert items(rows_of(start, n_rows, n_rows, disjoint=False), lens, each, kv_heads, nt, max_len) > have      # why the rule is there


def test_any_arrays_fit_the_workspace():
    r = random.Random(0)
    for _ in range(4000):
        group, kv_heads, n_rows, n_seqs = r.choice([1, 4, 8]), r.choice([1, 8, 40]), r.randint(1, 300), r.randint(1, 150)
        max_new, max_len = r.randint(1, n_rows), r.randint(24 * 64, 20000)
        nt = r.choice([1, 2, 8])
        start = [r.randint(-2, n_rows + 2) for _ in range(n_seqs + 1)]
        if r.random() < 0.4:
            start.sort()
        got = rows_of(start, n_rows, max_new)
        places = [x for r0, n in got for x in range(r0, r0 + n)]
        assert len(places) == len(set(places)) and all(0 <= x < n_rows for x in places)
        # items: whole tiles of all rows, and the cuts (the plan's bound)
        lens = [r.choice([r.randint(0, 100), max_len, r.randint(0, max_len), max_len + 5, -3]) for _ in range(n_seqs)]
        whole = (n_rows * group // (16 * nt) + min(n_seqs, n_rows)) * kv_heads
        most = ((max_len + 63) // 64 + 8) // 16
        assert items(got, lens, group, kv_heads, nt, max_len) <= min(whole + 4 * UNITS, whole * most)
