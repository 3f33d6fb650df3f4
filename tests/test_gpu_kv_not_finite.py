"""Infinities and NaN in V beside pages that are missing, and in keys that are cut into runs."""
import math

import pytest
import torch

import paper_2410_01028_amd as asd
from test_gpu_kv_ops import DEV, Pool, check_attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv", ["fp8", "bf16"])
def test_values_that_are_not_finite_beside_a_page_that_is_missing(kv):
    """NaN and infinities in the chunks in front of a page outside the pool, and behind it, that all rows of a tile see."""
    news, total = [64, 130, 200], [64, 1200, 200]
    p = Pool("bf16", kv, 40, 40, 128, 64, list(zip(news, total)), seed=23)
    k, v = p.normal(sum(total), 40, 128), p.normal(sum(total), 40, 128)
    at = total[0]                                        # the second sequence: key 0; the missing page holds its keys 640 .. 703
    v[at + 639, 3, 5], v[at + 580, 4, 6], v[at + 513, 5, 7], v[at + 704, 6, 8], v[at + 650, 7, 9] = math.nan, math.inf, -math.inf, math.nan, math.nan
    whole = p.batch(total, total)
    p.cache.append(whole, None, k, v)
    k, v = (torch.split(x, total) for x in p.cache.read(whole))
    whole.check()
    p.d_table[1, 10] = -1
    q = p.normal(sum(news), 40, 128)
    b = p.batch(news, total)
    out = p.cache.attend(b, q)
    with pytest.raises(asd.AsdError, match="pages"):
        b.check()
    keep = torch.cat([torch.arange(640), torch.arange(704, 1200)]).to(DEV)
    rows = slice(news[0], news[0] + news[1])
    check_attend(p, [130], [1136], q[rows], out[rows], [k[1][keep]], [v[1][keep]], 128 ** -0.5)
    assert bool(out[rows][:, 3, 5].isnan().all()) and bool(out[rows][:, 7, 9].isfinite().all())


@pytest.mark.parametrize("kv", ["fp8", "bf16"])
def test_values_that_are_not_finite_in_runs_of_many_rows(kv):
    """Keys that are cut into runs, for tiles of 128 rows: in chunks that all see, at the first and last keys of a run, in the chunks at the edge."""
    news, total = [300, 1, 90, 3], [9000, 40, 90, 2100]
    p = Pool("bf16", kv, 8, 2, 128, 256, list(zip(news, total)), seed=24)
    k, v = p.normal(sum(total), 2, 128), p.normal(sum(total), 2, 128)
    for i, key in enumerate((0, 63, 64, 1023, 1024, 2047, 3000, 5119, 8699, 8700, 8703, 8704, 8767, 8900, 8999)):
        v[key, i % 2, 3 * i] = (math.nan, math.inf, -math.inf)[i % 3]
    whole = p.batch(total, total)
    p.cache.append(whole, None, k, v)
    k, v = (torch.split(x, total) for x in p.cache.read(whole))
    b = p.batch(news, total)
    assert p.cache.attend_workspace(b) > 0
    q = p.normal(sum(news), 8, 128)
    out = p.cache.attend(b, q)
    b.check()
    check_attend(p, news, total, q, out, k, v, 128 ** -0.5)
