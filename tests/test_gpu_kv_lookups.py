"""Batches of shared beginnings with more sequences and groups than a wave looks at in one go (KVCache.attend_shared): groups that go over the borders of sixty-four, and thousands of them."""
import random

import pytest
import torch

import paper_2410_01028_amd as asd
from kv_spans_reference import HALF, close
from test_gpu_kv_ops import DEV, Pool
from test_gpu_kv_shared import Family, i32

pytestmark = pytest.mark.gpu

STARTS = {"long ones at the end of sixty-four": [*range(64), 300, *range(300, 363), 400], "empty ones": [0] * 100 + [5] * 70 + [130] * 130 + [400], "one for all": [0, 400],
          "sixty-fours": list(range(0, 400, 64)) + [400]}


@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
@pytest.mark.parametrize("kind", list(STARTS))
def test_groups_over_the_borders_of_what_a_wave_looks_at(kind, wide):
    r = random.Random(5)
    groups = []
    for f0, f1 in zip(STARTS[kind], STARTS[kind][1:]):
        shared = r.choice([64, 70, 128])
        groups.append((shared, [(1, shared + 1 + r.randrange(90)) for _ in range(f0, f1)]))
    f = Family("bf16", "fp8", 4, 2, 64, 64, groups, seed=51, wide=wide)
    assert f.start == STARTS[kind] and len(f.news) == 400
    q, b = f.p.normal(400, 4, 64, scale=2.0), f.p.batch(f.news, f.total)
    out = f.p.cache.attend_shared(b, f.groups, q)
    b.check()
    f.check(q, out)


@pytest.mark.parametrize("dtype,kv,cap", [("f32", "f32", 100), ("f32", "f32", 128), ("bf16", "fp8", 100), ("bf16", "fp8", 512)])
@pytest.mark.parametrize("each", [2, 256])
def test_thousands_of_sequences_and_groups(dtype, kv, cap, each):
    """One token of 8192 sequences, the first 64 of 100 tokens common to groups of `each`; with room for few tokens, and for so many that the shared keys are read apart."""
    n, total, shared, heads, h = 8192, 100, 64, 2, 32
    p = Pool(dtype, kv, heads, 1, h, 64, [(1, total)] * n, seed=52, max_len=cap)
    k, v = p.fill()
    first = torch.arange(n, device=DEV) // each * each
    p.d_table[:, 0] = p.d_table[first, 0]
    if cap > 128:
        p.d_table = torch.cat([p.d_table, torch.full((n, cap // 64 - 2), -1, dtype=torch.int32, device=DEV)], 1).contiguous()
    k, v = (torch.stack(x).double()[:, :, 0] for x in (k, v))
    k, v = (torch.cat([x[first, :shared], x[:, shared:]], 1) for x in (k, v))
    q, b = p.normal(n, heads, h, scale=2.0), p.batch([1] * n, [total] * n)
    groups = asd.KVGroups(i32(list(range(0, n + 1, each))), i32([shared] * (n // each)))
    out = p.cache.attend_shared(b, groups, q)
    b.check()
    # tolerances: kv_spans_reference.py
    weights = torch.softmax((q.double()[:, :, None] * k[:, None]).sum(-1) * h ** -0.5, -1)
    want, size = ((weights[..., None] * x[:, None]).sum(2) for x in (v, v.abs()))
    big = (q.double().abs()[:, :, None] * k.abs()[:, None]).sum(-1).amax(-1) * h ** -0.5
    e = 2 * h * 2.0 ** -24 * big[..., None] + 2.0 ** -20 + total * 2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0.0)
    close(out, want, size * e + (want.abs() + size * e) * HALF[dtype], "thousands of sequences")
