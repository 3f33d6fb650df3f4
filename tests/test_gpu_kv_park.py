"""An engine's sequence taken out into other pages and put back (Engine.park, Engine.resume) while another one uses the engine, and the
engine's own cache under the operators of KVCache."""
import numpy as np
import pytest
import torch

import asd_inputs as si
import paper_2410_01028_amd as asd
from kv_reference import attention, held
from test_gpu_parity import MID16

pytestmark = pytest.mark.gpu
TINY = si.SHAPES["tiny"]


def pools(shape, n_pages, page, kv_dtype):
    args = (shape.n_heads, shape.n_kv_heads, shape.head_dim, page, shape.dtype, kv_dtype)
    return [asd.KVCache(torch.full((n_pages * asd.kv_page_bytes(*args),), 0x7F, dtype=torch.uint8, device="cuda:0"), *args) for _ in range(shape.n_layers)]


@pytest.mark.parametrize("shape,ctx", [(TINY, 45), (MID16, 150)], ids=["tiny", "mid16"])
@pytest.mark.parametrize("bits8", [False, True], ids=["same type", "8 bits"])
def test_park_and_resume(shape, ctx, bits8):
    eng = asd.Engine(asd.make_config(shape, 256, page_tokens=64)).init_synthetic(3)
    eng.set_page_table([2, 0, 3, 1])
    toks = si.prompt(2, ctx + 8, shape.vocab)
    eng.prefill(toks[:ctx])
    want = eng.forward(toks[ctx:ctx + 3], ctx, commit=False)
    kv = [eng.get_kv(l, 0, ctx) for l in range(shape.n_layers)]
    caches = pools(shape, 5, 128, asd.DT_FP8 if bits8 else shape.dtype)      # pages of another size
    table = torch.tensor([[4, 1]], dtype=torch.int32, device="cuda:0")
    assert eng.park(caches, table) == ctx
    eng.prefill(si.prompt(9, 200, shape.vocab))                              # another conversation
    eng.resume(caches, table, ctx)
    assert eng.kv_len == ctx
    got = eng.forward(toks[ctx:ctx + 3], ctx, commit=False)
    back = [eng.get_kv(l, 0, ctx) for l in range(shape.n_layers)]
    if not bits8:
        assert np.array_equal(got["logits"], want["logits"]) and np.array_equal(got["cos"], want["cos"])
    for (k, v), (k1, v1) in zip(kv, back):
        for x, y in ((k, k1), (v, v1)):
            assert np.array_equal(y, held(torch.from_numpy(x).double())[0].float().numpy() if bits8 else x)
    with pytest.raises(asd.AsdError):
        eng.resume(caches, table, 257)
    with pytest.raises(asd.AsdError):
        eng.park(caches[1:], table)
    with pytest.raises(asd.AsdError):
        eng.kv_cache(shape.n_layers)
    eng.close()


def test_the_engines_cache_under_attend():
    """New rows attend to what an engine's prompt pass has left in its pages."""
    eng = asd.Engine(asd.make_config(TINY, 128, page_tokens=64)).init_synthetic(0)
    eng.set_page_table([1, 0])
    eng.prefill(si.prompt(0, 100, TINY.vocab))
    k, v = (torch.from_numpy(x).cuda() for x in eng.get_kv(2, 0, 100))
    cache, table = eng.kv_cache(2)
    b = asd.KVBatch(table, torch.tensor([0, 3], dtype=torch.int32, device="cuda:0"), torch.tensor([100], dtype=torch.int32, device="cuda:0"), 3, 3, 128)
    q = torch.randn(3, TINY.n_heads, TINY.head_dim, generator=torch.Generator("cuda:0").manual_seed(1), device="cuda:0")
    out = cache.attend(b, q)
    b.check()
    want, size, big = attention(q, k, v, 97, TINY.head_dim ** -0.5)
    # (tolerance as in test_gpu_kv_ops.py)
    e = 2 * TINY.head_dim * 2.0 ** -24 * big[..., None] + 2.0 ** -20 + 100 * 2.0 ** -24
    assert bool(((out.double() - want).abs() <= size * e + want.abs() * 2.0 ** -24).all())
    eng.close()


def test_a_sequence_that_cannot_be_put_back():
    """A page table that leads out of the pool, or does not reach far enough: the engine's pages may hold parts of two sequences then, so it has none.
    Where nothing was begun, its own stays."""
    eng = asd.Engine(asd.make_config(TINY, 256, page_tokens=64)).init_synthetic(3)
    caches = pools(TINY, 2, 64, TINY.dtype)
    table = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda:0")
    toks = si.prompt(2, 100, TINY.vocab)
    eng.prefill(toks)
    want = eng.get_kv(1, 0, 100)
    assert eng.park(caches, table) == 100
    for bad in (caches[1:], caches + caches[:1]):
        with pytest.raises(asd.AsdError):
            eng.resume(bad, table, 100)
        assert eng.kv_len == 100
    with pytest.raises(asd.AsdError, match="pages"):
        eng.resume(caches, torch.tensor([[1, 2]], dtype=torch.int32, device="cuda:0"), 100)
    assert eng.kv_len == 0
    with pytest.raises(asd.AsdError, match="lengths"):
        eng.resume(caches, table, 129)
    assert eng.kv_len == 0
    eng.resume(caches, table, 100)
    assert eng.kv_len == 100
    got = eng.get_kv(1, 0, 100)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    eng.close()
