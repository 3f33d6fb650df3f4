"""KVCache.attend_shared: values of all rows where sequences are in no group, and where rows or lengths are out of range.  Tolerances: kv_spans_reference.py."""
import pytest
import torch

import paper_2410_01028_amd as asd
from kv_spans_reference import check, in_window
from test_gpu_kv_ops import COMBOS, DEV, Pool
from test_gpu_kv_shared import Family, i32, widen
from test_kv_spans_split import mended

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
@pytest.mark.parametrize("dtype,kv", COMBOS)
@pytest.mark.parametrize("start,shared", [([1, 3], [200]), ([1, 3, 3], [200, 9]), ([1, 3, 3, 3], [200, 9, 7]), ([1, 3, 4, 6], [200, 50, 64]), ([1, 1, 3], [5, 200]), ([0, 0, 1, 3, 3, 6], [3, 100, 200, 1, 0])])
def test_sequences_in_no_group(dtype, kv, start, shared, wide):
    """Sequences in front of, between and behind the groups take their own pages, as do those of a group that shares nothing."""
    f = Family(dtype, kv, 8, 2, 64, 64, [(100, [(1, 130)]), (200, [(2, 202), (1, 300)]), (50, [(3, 80)]), (64, [(1, 90), (1, 70)])], seed=6, wide=wide)
    q, b = f.p.normal(sum(f.news), 8, 64, scale=2.0), f.p.batch(f.news, f.total)
    out = f.p.cache.attend_shared(b, asd.KVGroups(i32(start), i32(shared)), q)
    b.check()
    f.check(q, out)


@pytest.mark.parametrize("start,lens", [([0, 3, 1, 6, 8], [200, 210, 220, 230]), ([0, 2, 4, 6, 2 ** 31 - 1], [200, 200, 200, 200]), ([-9, 2, 4, 6, 8], [200, 200, 200, 200]),
                                        ([0, 8, 0, 8, 8], [200, 200, 200, 200]), ([0, 2, 4, 6, 8], [2 ** 31 - 1, 1, -3, 200]), ([5, 4, 3, 2, 1], [200, 200, 200, 200]),
                                        ([0, 2, 4, 6, 9], [131, 132, 65, 66]), ([0, 2, 4, 3, 8], [240, 135, 240, 100])])
@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
@pytest.mark.parametrize("dtype,kv", [("bf16", "fp8"), ("f32", "f32")])
def test_rows_out_of_range(dtype, kv, start, lens, wide):
    """Sequences that hold all their tokens, the common ones too, in pages of their own: rows that are left keep their positions and see what lies in front of them, the others stay as they are."""
    p = Pool(dtype, kv, 8, 2, 64, 64, [(1, 240)] * 4, seed=61)
    if wide:
        widen(p)
    common = [p.normal(130, 2, 64) for _ in range(2)]
    own = [[p.normal(240, 2, 64) for _ in range(4)] for _ in range(2)]
    k, v = ([torch.cat([x[:n], y[n:]]) for y, n in zip(ys, (130, 130, 64, 64))] for x, ys in zip(common, own))
    whole = p.batch([240] * 4, [240] * 4)
    p.cache.append(whole, None, torch.cat(k), torch.cat(v))
    k, v = (torch.split(x, 240) for x in p.cache.read(whole))
    cap = p.cap if wide else 240
    b = asd.KVBatch(p.d_table, i32(start), i32(lens), 8, 3, cap)
    q = p.normal(8, 8, 64, scale=2.0)
    out = p.cache.attend_shared(b, asd.KVGroups(i32([0, 2, 4]), i32([130, 64])), q, out=torch.full_like(q, 7.0))
    with pytest.raises(asd.AsdError, match="rows or lengths"):
        b.check()
    left = torch.ones(8, dtype=torch.bool)
    for i, (r0, n, first, length) in enumerate(mended(start, lens, 8, 3, cap)):
        if not n:
            continue
        left[r0:r0 + n] = False
        rows = slice(r0, r0 + n)
        pos, length = torch.arange(first, first + n, device=DEV), max(length, 1)        # (no token: rows that see nothing of one)
        check(dtype, q[rows], out[rows], k[i][:length], v[i][:length], in_window(pos, length, 2 ** 30, 0), 0.125, f"sequence {i}")
    assert bool((out[left.to(DEV)] == 7.0).all())


@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
@pytest.mark.parametrize("dtype,kv", COMBOS)
@pytest.mark.parametrize("groups", [[(333, [(0, 333), (1, 340), (1, 500), (1, 334)])], [(200, [(0, 900), (5, 300), (3, 203)]), (64, [(0, 64), (0, 100), (2, 66)])],
                                    [(130, [(0, 130), (70, 210), (40, 170), (1, 131)])], [(1000, [(0, 1000)] + [(1, 1001 + 7 * i) for i in range(40)])]],
                         ids=["tokens", "drafts", "chunks", "many"])
def test_common_tokens_that_are_a_sequence_of_their_own(dtype, kv, groups, wide):
    """A system prompt kept as a sequence without new rows; the page tables of the others say nothing of its pages."""
    f = Family(dtype, kv, 16, 2, 64, 64, groups, seed=62, wide=wide)
    for i, first in enumerate(f.first):
        if i != first:
            f.p.d_table[i, :f.shared[i] // 64] = torch.tensor([-1, 2 ** 31 - 1, f.p.cache.n_pages, -2 ** 31], dtype=torch.int32, device=DEV).repeat(10)[:f.shared[i] // 64]
    q, b = f.p.normal(sum(f.news), 16, 64, scale=2.0), f.p.batch(f.news, f.total)
    out = f.p.cache.attend_shared(b, f.groups, q)
    b.check()
    f.check(q, out)


@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
def test_a_padded_batch(wide):
    """Captured for eight places of which three to eight are taken; the others have no rows and no tokens, and lie in the last group or in none."""
    f = Family("bf16", "fp8", 16, 2, 64, 64, [(200, [(1, 201 + 9 * i) for i in range(8)])], seed=63, wide=wide)
    q = f.p.normal(8, 16, 64)
    out, b = torch.empty_like(q), f.p.batch(f.news, f.total)
    groups = asd.KVGroups(i32([0, 8]), i32([200]))
    ws = torch.empty(max(f.p.cache.attend_shared_workspace(b, groups), 256), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f.p.cache.attend_shared(b, groups, q, out=out, workspace=ws)
    for taken, end in ((8, 8), (3, 8), (5, 5), (8, 8), (3, 3)):
        b.row_start.copy_(torch.tensor([min(i, taken) for i in range(9)]))
        b.kv_len.copy_(torch.tensor(f.total[:taken] + [0] * (8 - taken)))
        groups.group_start[1] = end
        out.fill_(7.0)
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        b.check()
        for i in range(taken):
            check("bf16", q[i:i + 1], out[i:i + 1], f.k[i], f.v[i], in_window(torch.tensor([f.total[i] - 1], device=DEV), f.total[i], 2 ** 30, 0), 0.125, f"{taken} taken, sequence {i}")
        assert bool((out[taken:] == 7.0).all())
