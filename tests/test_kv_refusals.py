"""Refusals of the operators over a paged cache of several sequences: all of them happen on the host, before a device is needed."""
import ctypes

import pytest

import paper_2410_01028_amd as asd

P = 1 << 20       # an aligned address that no call reads


def shape(**kw):
    a = dict(n_heads=8, n_kv_heads=2, head_dim=64, page_tokens=64, dtype=asd.DT_BF16, kv_dtype=asd.DT_FP8) | kw
    return asd.KvShape(*a.values())


def batch(**kw):
    a = dict(pages=P, page_table=P, row_start=P, kv_len=P, status=None, n_pages=4, table_stride=2, n_seqs=2, n_rows=6, max_new=3, max_len=100) | kw
    return asd.KvBatch(*a.values())


def call(name, s, b, **kw):
    L = asd._kv_lib()
    s, b = (None if x is None else ctypes.addressof(x) for x in (s, b))
    a = dict(q=P, qs=512, k=P, ks=128, v=P, vs=128, out=P, os=512, scale=0.125, ws=P, wb=1 << 40,
             prep=asd.KvPrep(None, None, 1e-5, P, 10, 64, 0)) | kw
    if name == "append":
        rc = L.asd_kv_append(s, b, None if a["prep"] is None else ctypes.addressof(a["prep"]), a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["out"], a["os"], None)
    elif name == "attend":
        rc = L.asd_kv_attend(s, b, a["q"], a["qs"], a["out"], a["os"], a["scale"], a["ws"], a["wb"], None)
    else:
        rc = L.asd_kv_read(s, b, a["k"], a["ks"], a["v"], a["vs"], None)
    return rc, asd.lib().asd_last_error(None).decode()


@pytest.mark.parametrize("kw", [dict(n_heads=7), dict(n_kv_heads=0), dict(head_dim=96), dict(head_dim=256), dict(page_tokens=32), dict(page_tokens=0),
                                dict(dtype=asd.DT_FP8), dict(dtype=5), dict(kv_dtype=asd.DT_F32), dict(kv_dtype=-1), dict(n_heads=8192, n_kv_heads=8192)])
def test_shapes(kw):
    assert asd._kv_lib().asd_kv_page_bytes(ctypes.byref(shape(**kw))) == 0
    for name in ("append", "attend", "read"):
        assert call(name, shape(**kw), batch())[0] == asd.E_INVAL
    s, b = shape(**kw), batch()
    assert asd._kv_lib().asd_kv_attend_workspace(ctypes.addressof(s), ctypes.addressof(b)) == 0
    assert call("attend", None, batch())[0] == asd.E_INVAL


@pytest.mark.parametrize("kw,text", [(dict(pages=None), "pages"), (dict(pages=P + 8), "pages"), (dict(page_table=None), "page_table"), (dict(kv_len=P + 2), "aligned"),
                                     (dict(n_pages=0), "n_pages"), (dict(table_stride=0), "table_stride"), (dict(n_seqs=0), "n_seqs"), (dict(n_seqs=70000), "n_seqs"),
                                     (dict(n_rows=0), "n_rows"), (dict(n_rows=1 << 29), "n_rows"), (dict(max_new=0), "max_new"), (dict(max_new=7), "max_new"),
                                     (dict(max_len=0), "max_len"), (dict(max_len=1 << 25), "max_len")])
def test_batches(kw, text):
    for name in ("append", "attend", "read"):
        rc, why = call(name, shape(), batch(**kw))
        assert rc == asd.E_INVAL and text in why and name in why
    assert call("read", shape(), None)[0] == asd.E_INVAL


@pytest.mark.parametrize("name,kw", [("append", dict(k=None)), ("append", dict(v=None)), ("append", dict(out=None)), ("append", dict(q=None)), ("append", dict(prep=None)),
                                     ("append", dict(k=P + 8)), ("append", dict(ks=127)), ("append", dict(ks=64)), ("append", dict(qs=504)), ("append", dict(os=-512)),
                                     ("append", dict(prep=asd.KvPrep(None, None, 0, P, 10, 12, 0))), ("append", dict(prep=asd.KvPrep(None, None, 0, P, 10, 72, 0))), ("append", dict(prep=asd.KvPrep(None, None, 0, P, 10, 24, 0))),
                                     ("append", dict(prep=asd.KvPrep(None, None, 0, None, 10, 64, 0))), ("append", dict(prep=asd.KvPrep(None, None, 0, P, 0, 64, 0))),
                                     ("append", dict(prep=asd.KvPrep(P + 4, None, 0, P, 10, 64, 0))), ("append", dict(prep=asd.KvPrep(P, P, -1.0, P, 10, 64, 0))),
                                     ("append", dict(prep=asd.KvPrep(P, P, float("nan"), P, 10, 64, 0))),
                                     ("attend", dict(q=None)), ("attend", dict(out=None)), ("attend", dict(qs=500)), ("attend", dict(out=P + 2)),
                                     ("attend", dict(scale=0.0)), ("attend", dict(scale=float("nan"))), ("attend", dict(scale=float("inf"))), ("attend", dict(scale=-1.0)),
                                     ("read", dict(k=P + 4)), ("read", dict(vs=64))])
def test_buffers(name, kw):
    rc, why = call(name, shape(), batch(), **kw)
    assert rc == asd.E_INVAL and name in why


def test_workspace():
    big = batch(max_len=5000, table_stride=100)
    s = shape()
    need = asd._kv_lib().asd_kv_attend_workspace(ctypes.addressof(s), ctypes.addressof(big))
    assert need > 0
    assert call("attend", shape(), big, wb=need - 1)[0] == asd.E_NOMEM
    assert call("attend", shape(), big, ws=None)[0] == asd.E_INVAL
    assert call("attend", shape(), big, ws=P + 16)[0] == asd.E_INVAL


@pytest.mark.parametrize("kw", [dict(kind=4), dict(kind=-1), dict(rot_dim=12), dict(rot_dim=0), dict(rot_dim=136), dict(theta=1.0), dict(theta=float("nan")), dict(kind=1, factor=0.5),
                                dict(kind=2, low=4.0, high=4.0), dict(kind=3, low=0.0), dict(kind=3, trained=0.0), dict(gain=-1.0), dict(gain=float("nan"))])
def test_rope_tables(kw):
    a = dict(kind=0, rot_dim=64, theta=1e4, factor=2.0, low=1.0, high=4.0, trained=4096.0, gain=1.0) | kw
    assert asd._kv_lib().asd_rope_table(asd.Rope(*a.values()), 10, P, None) == asd.E_INVAL
    assert b"asd_rope_table" in asd.lib().asd_last_error(None)
    ok = asd.Rope(0, 64, 1e4, 2.0, 1.0, 4.0, 4096.0, 1.0)
    for positions, table in ((0, P), (1 << 25, P), (10, None), (10, P + 4)):
        assert asd._kv_lib().asd_rope_table(ok, positions, table, None) == asd.E_INVAL


def test_engine_calls_without_an_engine():
    L = asd._kv_lib()
    assert L.asd_kv_view(None, 0, asd.KvShape(), asd.KvBatch()) == asd.E_INVAL
    assert L.asd_set_kv_len(None, 0) == asd.E_INVAL


def test_a_table_is_told_from_one_of_its_rows():
    """A rotary table has three dimensions: with one row of it, the kernels would take its pairs for positions."""
    import torch
    cache = asd.KVCache.__new__(asd.KVCache)
    cache.__dict__.update(_torch=torch, _index=-1, device=torch.device("cpu"))       # (-1: a CPU tensor's device)
    table = torch.zeros(10, 32, 2)
    assert cache._floats("rope", table, None, 32, 2) == table.data_ptr()
    for bad in (table[3], table[None], table.double(), table[:, :16], table[:, ::2]):
        with pytest.raises(asd.AsdError):
            cache._floats("rope", bad, None, 32, 2)
    with pytest.raises(asd.AsdError):
        cache._floats("q_gain", torch.zeros(2, 64), 64)


@pytest.mark.parametrize("kind,names", [(asd.KVBatch, ("page_table", "row_start", "kv_len", "status", "n_rows", "max_new", "max_len")),
                                        (asd.KVCache, ("pages", "n_pages", "n_heads", "n_kv_heads", "head_dim", "torch_dtype"))])
def test_what_calls_rely_on_does_not_change(kind, names):
    """Calls pass addresses and bounds that were taken when the object was made: another tensor or bound in its place is refused."""
    x = kind.__new__(kind)
    for name in names:
        setattr(x, name, 1)
        with pytest.raises(AttributeError):
            setattr(x, name, 2)
        assert getattr(x, name) == 1


@pytest.mark.parametrize("name", ["append", "attend"])
def test_launches_that_no_card_takes(name):
    """65536 tokens of as many sequences with 4096 heads: more than 2^32 threads, and a launch's number of them must fit 32 bits."""
    s, b = shape(n_heads=4096, n_kv_heads=4096, head_dim=32), batch(n_seqs=65536, n_rows=65536, max_new=1)
    rc, why = call(name, s, b, qs=4096 * 32, ks=4096 * 32, vs=4096 * 32, os=4096 * 32, prep=asd.KvPrep(None, None, 0, P, 10, 32, 0))
    assert rc == asd.E_INVAL and name in why and "too large" in why


def test_a_read_that_no_card_takes():
    rc, why = call("read", shape(n_heads=1, n_kv_heads=1, head_dim=32), batch(n_rows=(1 << 31) - 1), ks=32, vs=32)
    assert rc == asd.E_INVAL and "too large" in why


def test_a_scale_that_overflows():
    """scale * log2(e) is what the kernels multiply by: it must be a number, too."""
    rc, why = call("attend", shape(), batch(), scale=3e38)
    assert rc == asd.E_INVAL and "scale" in why
