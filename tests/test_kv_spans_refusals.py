"""Refusals of the attention with a window and of the attention of sequences that begin with the same tokens: on the host, before a device is needed."""
import ctypes

import pytest

import paper_2410_01028_amd as asd
from test_kv_refusals import P, batch, shape


def groups(**kw):
    a = dict(group_start=P, shared_len=P, n_groups=2) | kw
    return asd.KvGroups(*a.values())


def call(name, s, b, **kw):
    L = asd._kv_lib()
    a = dict(q=P, qs=512, out=P, os=512, scale=0.125, ws=P, wb=1 << 40, window=16, sinks=2, groups=groups()) | kw
    form = (a["window"], a["sinks"]) if name == "attend_window" else (None if a["groups"] is None else ctypes.addressof(a["groups"]),)
    s, b = (None if x is None else ctypes.addressof(x) for x in (s, b))
    rc = getattr(L, f"asd_kv_{name}")(s, b, *form, a["q"], a["qs"], a["out"], a["os"], a["scale"], a["ws"], a["wb"], None)
    need = getattr(L, f"asd_kv_{name}_workspace")(s, b, *form)
    return rc, asd.lib().asd_last_error(None).decode(), need


NAMES = ("attend_window", "attend_shared")


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("kw", [dict(n_heads=7), dict(head_dim=96), dict(page_tokens=32), dict(dtype=asd.DT_FP8), dict(kv_dtype=asd.DT_F32)])
def test_shapes(name, kw):
    rc, why, need = call(name, shape(**kw), batch())
    assert rc == asd.E_INVAL and name in why and need == 0
    assert call(name, None, batch())[0] == asd.E_INVAL and call(name, shape(), None)[0] == asd.E_INVAL


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("kw,text", [(dict(pages=None), "pages"), (dict(page_table=None), "page_table"), (dict(kv_len=P + 2), "aligned"), (dict(n_pages=0), "n_pages"),
                                     (dict(n_seqs=70000), "n_seqs"), (dict(n_rows=1 << 29), "n_rows"), (dict(max_new=7), "max_new"), (dict(max_len=1 << 25), "max_len")])
def test_batches(name, kw, text):
    rc, why, need = call(name, shape(), batch(**kw))
    assert rc == asd.E_INVAL and text in why and name in why and need == 0


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("kw", [dict(q=None), dict(out=None), dict(qs=500), dict(os=64), dict(out=P + 2), dict(scale=0.0), dict(scale=float("nan")), dict(scale=3e38)])
def test_buffers(name, kw):
    rc, why, _ = call(name, shape(), batch(), **kw)
    assert rc == asd.E_INVAL and name in why


@pytest.mark.parametrize("kw", [dict(window=0), dict(window=-5), dict(sinks=-1), dict(window=-2 ** 31, sinks=-2 ** 31)])
def test_windows(kw):
    rc, why, need = call("attend_window", shape(), batch(), **kw)
    assert rc == asd.E_INVAL and ("window" in why or "sinks" in why) and need == 0


@pytest.mark.parametrize("kw", [dict(group_start=None), dict(shared_len=None), dict(group_start=P + 2), dict(shared_len=P + 1), dict(n_groups=0), dict(n_groups=-1), dict(n_groups=65537)])
def test_groups(kw):
    rc, why, need = call("attend_shared", shape(), batch(), groups=groups(**kw))
    assert rc == asd.E_INVAL and "group" in why and need == 0
    assert call("attend_shared", shape(), batch(), groups=None)[0] == asd.E_INVAL


@pytest.mark.parametrize("name", NAMES)
def test_workspace(name):
    big = batch(max_len=5000, table_stride=100)
    kw = dict(window=4000)
    need = call(name, shape(), big, ws=None, **kw)[2]
    assert need > 0
    assert call(name, shape(), big, wb=need - 1, **kw)[0] == asd.E_NOMEM
    assert call(name, shape(), big, ws=None, **kw)[0] == asd.E_INVAL
    assert call(name, shape(), big, ws=P + 16, **kw)[0] == asd.E_INVAL


@pytest.mark.parametrize("name", NAMES)
def test_batches_whose_launch_is_too_large(name):
    rc, why, _ = call(name, shape(n_heads=4096, n_kv_heads=4096, head_dim=32), batch(n_seqs=65536, n_rows=(1 << 19) - 1, max_new=1), qs=1 << 20, os=1 << 20, wb=1 << 62)
    assert rc == asd.E_INVAL and "too large" in why
