"""Cache memory that was never written beside the keys that rows see: pages that start as 0xFF bytes (NaN as numbers and as codes, infinity as a scale), in which only what some row
sees has been appended.  Against 64 bits; tolerances: kv_spans_reference.py."""
import functools

import pytest
import torch

import test_gpu_kv_shared as shared
from kv_spans_reference import check, in_window
from test_gpu_kv_ops import COMBOS, DEV, Pool

pytestmark = pytest.mark.gpu

# rows and tokens of sequences, heads, KV heads, head dim
KINDS = {"tokens": ([1, 1, 1], [700, 1300, 65], 8, 2, 64), "drafts": ([6, 5, 1], [900, 600, 300], 8, 2, 128), "chunks": ([30, 17, 1], [900, 600, 300], 8, 2, 64),
         "many": ([130, 300, 70], [1301, 900, 1000], 40, 40, 64), "many, groups of heads": ([130, 300, 70], [1301, 900, 1000], 64, 8, 128)}


@pytest.mark.parametrize("dtype,kv", COMBOS)
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("window,sinks", [(100, 4), (333, 70), (64, 64), (250, 0), (700, 200), (1, 1)])
def test_only_first_tokens_and_windows_are_written(dtype, kv, kind, window, sinks):
    """Of each sequence only its first tokens and the windows of its rows are in the cache: their ends lie inside chunks, in one chunk for some."""
    news, total, heads, kv_heads, h = KINDS[kind]
    p = Pool(dtype, kv, heads, kv_heads, h, 64, list(zip(news, total)), seed=41, fill=0xFF)
    first = [max(0, t - n - window + 1) for n, t in zip(news, total)]                       # the first row's window
    head = [min(sinks, f) for f in first]
    parts = []
    for rows, lens in ((head, head), ([t - f for f, t in zip(first, total)], total)):
        if not sum(rows):
            parts.append([torch.empty(0, kv_heads, h, dtype=p.t, device=DEV)] * 6)
            continue
        b = p.batch(rows, lens)
        p.cache.append(b, None, p.normal(sum(rows), kv_heads, h), p.normal(sum(rows), kv_heads, h))
        k, v = p.cache.read(b)
        b.check()
        parts.append([x for y in (k, v) for x in torch.split(y, rows)])
    q, b = p.normal(sum(news), heads, h, scale=2.0), p.batch(news, total)
    out = p.cache.attend_window(b, q, window, sinks)
    b.check()
    at = 0
    for i, (n, t) in enumerate(zip(news, total)):
        k, v = (torch.cat([parts[0][j][:head[i]], parts[1][j]]) for j in (i, 3 + i))
        keys = torch.cat([torch.arange(head[i], device=DEV), torch.arange(first[i], t, device=DEV)])
        seen = in_window(torch.arange(t - n, t, device=DEV), t, window, sinks)[:, keys]
        check(dtype, q[at:at + n], out[at:at + n], k, v, seen, h ** -0.5, f"sequence {i}")
        at += n


@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
@pytest.mark.parametrize("dtype,kv", COMBOS)
@pytest.mark.parametrize("kv_heads,kind", [(2, "samples"), (2, "drafts"), (64, "requests"), (2, "alone")])
def test_only_shared_and_own_tokens_are_written(monkeypatch, dtype, kv, kv_heads, kind, wide):
    """Sequences that leave their common tokens inside a page: their own pages hold nothing in front of that place, the first one's nothing of theirs behind it."""
    monkeypatch.setattr(shared, "Pool", functools.partial(Pool, fill=0xFF))
    f = shared.Family(dtype, kv, 2 * kv_heads, kv_heads, 64, 64, shared.FAMILIES[kind], seed=42, wide=wide)
    q, b = f.p.normal(sum(f.news), 2 * kv_heads, 64, scale=2.0), f.p.batch(f.news, f.total)
    out = f.p.cache.attend_shared(b, f.groups, q)
    b.check()
    f.check(q, out)


@pytest.mark.parametrize("dtype,kv", COMBOS)
@pytest.mark.parametrize("kind", list(KINDS))
def test_nothing_is_written_behind_the_last_token(dtype, kv, kind):
    news, total, heads, kv_heads, h = KINDS[kind]
    p = Pool(dtype, kv, heads, kv_heads, h, 128, list(zip(news, total)), seed=43, fill=0xFF)
    k, v = p.fill()
    q, b = p.normal(sum(news), heads, h, scale=2.0), p.batch(news, total)
    for out, window, sinks in ((p.cache.attend(b, q), 2 ** 30, 0), (p.cache.attend_window(b, q, 200, 5), 200, 5)):
        b.check()
        at = 0
        for i, (n, t) in enumerate(zip(news, total)):
            check(dtype, q[at:at + n], out[at:at + n], k[i], v[i], in_window(torch.arange(t - n, t, device=DEV), t, window, sinks), h ** -0.5, f"sequence {i}, window {window}")
            at += n
