"""Batches whose rows and lengths lead past the bounds that they were given."""
import pytest
import torch

import paper_2410_01028_amd as asd
from test_gpu_kv_ops import DEV, Pool, check_attend
from test_kv_split import rows_of

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def batch(p, start, lens, n_rows, max_new, max_len=None):
    return asd.KVBatch(p.d_table, i32(start), i32(lens), n_rows, max_new, max_len or p.cap)


def places(start, lens, n_rows, max_new, cap):
    """(first row, rows, position of the first) of every sequence: its first max_new rows inside the buffers, at the positions that the arrays
    give them, up to cap."""
    out = []
    for (r0, n), f1, length in zip(rows_of(start, n_rows, max_new), start[1:], lens):
        first = length - f1 + r0
        out.append((r0, max(0, min(n, cap - first)), first))
    return out


# row_start, lengths, rows, most new rows, most tokens
BEYOND = {"a token too far": ([0, 1, 2, 3], [257, 100, 256], 3, 1, 256),
          "past the bound, not the table": ([0, 4, 7], [203, 200], 7, 4, 200),
          "rows at the end and behind it": ([0, 4, 5, 9], [258, 1, 1000], 9, 4, 256),
          "more rows than max_new": ([0, 70, 76, 77], [150, 200, 3], 80, 4, 256),
          "rows behind the buffers": ([0, 2, 40], [90, 130], 30, 28, 256),
          "rows in front of the buffers": ([-5, 6, 8], [90, 130], 8, 8, 256),
          "far away": ([0, 3, 6, 9], [2 ** 31 - 1, -2 ** 31, 256], 9, 3, 256),
          "rows far away": ([-2 ** 31, 3, 2 ** 31 - 1], [100, 2 ** 31 - 1], 9, 9, 256)}


@pytest.mark.parametrize("dtype,kv", [("bf16", "fp8"), ("f32", "f32")])
@pytest.mark.parametrize("kind", list(BEYOND))
def test_a_row_keeps_its_place(kind, dtype, kv):
    """What is cut does not move the rows that are left: they are written, attend and are read back at their own positions, and nothing else is touched."""
    start, lens, n_rows, max_new, max_len = BEYOND[kind]
    p, ref = (Pool(dtype, kv, 4, 2, 64, 64, [(0, 256)] * len(lens), seed=22) for _ in range(2))
    p.fill()
    ref.pages.copy_(p.pages)
    b = batch(p, start, lens, n_rows, max_new, max_len)
    x = [p.normal(n_rows, heads, 64) for heads in (4, 2, 2)]
    seven = [torch.full_like(t, 7.0) for t in x]
    turned = p.cache.append(b, *x, q_out=seven[0].clone())
    with pytest.raises(asd.AsdError, match="rows or lengths"):
        b.check()
    got_k, got_v = p.cache.read(b, seven[1].clone(), seven[2].clone())
    out = p.cache.attend(b, x[0], out=seven[0].clone())
    want = [t.clone() for t in (seven[0], seven[1], seven[2], seven[0])]
    none = torch.ones(n_rows, dtype=torch.bool, device=DEV)      # rows that are nowhere
    for i, (r0, n, first) in enumerate(places(start, lens, n_rows, max_new, max_len)):
        lead = min(max(-first, 0), n)                    # in front of position 0
        if n:
            none[r0:r0 + n] = False
        if n == lead:
            continue
        rows = slice(r0 + lead, r0 + n)
        one = asd.KVBatch(ref.d_table[i:i + 1].contiguous(), i32([0, n - lead]), i32([first + n]), n - lead, n - lead, 256)
        want[0][rows] = ref.cache.append(one, *(t[rows].contiguous() for t in x))
        want[1][rows], want[2][rows] = ref.cache.read(one)
        want[3][rows] = ref.cache.attend(one, x[0][rows].contiguous())
        one.check()
        assert bool((out[r0:r0 + lead] == 0).all())
        k, v = ref.cache.read(asd.KVBatch(ref.d_table[i:i + 1].contiguous(), i32([0, first + n]), i32([first + n]), first + n, first + n, 256))
        check_attend(p, [n - lead], [first + n], x[0][rows], out[rows], [k], [v], 0.125)
        want[3][r0 + lead:r0 + n] = out[rows]
        want[3][r0:r0 + lead] = 0.0
    assert torch.equal(p.pages, ref.pages)
    for a, w in zip((turned, got_k, got_v), want):
        assert torch.equal(a, w)
    assert bool((out[none] == 7.0).all())
