"""Numbers that the library takes in 32 bits: ones that do not fit are refused by the binding, not cut to their low bits."""
import pytest
import torch

import paper_2410_01028_amd as asd

BIG = 1 << 32


@pytest.mark.parametrize("place", range(6))
def test_shapes(place):
    args = [8, 2, 64, 64, asd.DT_BF16, asd.DT_FP8]
    assert asd.kv_page_bytes(*args) > 0
    args[place] += BIG
    with pytest.raises(asd.AsdError, match="32 bits"):
        asd.kv_page_bytes(*args)
    with pytest.raises(asd.AsdError, match="32 bits"):
        asd.KVCache(torch.zeros(1, dtype=torch.uint8), *args)


@pytest.mark.parametrize("name", ["n_rows", "max_new", "max_len"])
def test_batches(name):
    i32 = lambda *shape: torch.zeros(*shape, dtype=torch.int32)      # noqa: E731
    bounds = dict(n_rows=2, max_new=2, max_len=10)
    for value in (BIG + 10, -BIG + 10, 1 << 31):
        with pytest.raises(asd.AsdError, match=f"{name}.*32 bits"):
            asd.KVBatch(i32(1, 1), i32(2), i32(1), **bounds | {name: value})


@pytest.mark.parametrize("kw", [dict(rot_dim=BIG + 64), dict(positions=BIG + 10), dict(kind=BIG)])
def test_rope_tables(kw):
    with pytest.raises(asd.AsdError, match="32 bits"):
        asd.rope_table(**dict(rot_dim=64, positions=10, device="cuda:0") | kw)


def test_rotated_dims():
    cache = asd.KVCache.__new__(asd.KVCache)
    cache.__dict__.update(head_dim=64)
    for rot_dim in (BIG, BIG + 64, 72, -BIG):
        with pytest.raises(asd.AsdError, match="rot_dim"):
            cache.append(None, None, None, None, rot_dim=rot_dim)
