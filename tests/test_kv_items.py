"""The kernels of the attention with a window and of shared beginnings carried out on the CPU (kv_items_on_cpu.cpp) but for the work on a tile: whatever the arrays hold, every row that
belongs to a sequence is answered once, from sums that its own items have left inside the workspace and that cover the chunks its tile walks; and how the look-ups grow."""
import ctypes
import os
import random
import re
import shutil
import subprocess

import numpy as np
import pytest

import paper_2410_01028_amd as asd
from test_kv_spans_split import mended

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2410_01028_amd", "csrc")
GUARD = 4096


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    hipcc = shutil.which("hipcc")
    if not hipcc:
        pytest.skip("no hipcc")
    tmp = tmp_path_factory.mktemp("items")
    text = open(os.path.join(CSRC, "asd_kv_spans.hip")).read()
    text, n = re.subn(r"(kv_\w+<[^;<>]*>)<<<(.+?), 256, 0, stream>>>\((.*?)\);", r"on_cpu([&] { \1(\3); }, \2);", text)
    assert n >= 8 and "<<<" not in text
    text = re.sub(r'#include "(.*?)"', lambda m: f'#include "{CSRC}/{m[1]}"', text)
    (tmp / "spans.inc").write_text(text)
    out = str(tmp / "items.so")
    subprocess.run([hipcc, "--offload-arch=gfx950", "--cuda-host-only", "-std=c++17", "-O2", "-fPIC", "-shared", "-w", f'-DSPANS="{tmp}/spans.inc"', "-x", "hip",
                    os.path.join(HERE, "kv_items_on_cpu.cpp"), "-o", out], check=True, timeout=600)
    L = ctypes.CDLL(out)
    vp, i64, i32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
    L.cpu_begin.argtypes = [vp, sz, i32, i32, i32, i64]
    L.cpu_fault.restype = ctypes.c_char_p
    L.cpu_answered.restype = L.cpu_lows.restype = vp
    L.cpu_lows.argtypes = [i32]
    L.cpu_counts.argtypes = [vp]
    L.asd_kv_attend_window_workspace.restype = L.asd_kv_attend_shared_workspace.restype = sz
    L.asd_kv_attend_window_workspace.argtypes = [vp, vp, i32, i32]
    L.asd_kv_attend_window.argtypes = [vp, vp, i32, i32, vp, i64, vp, i64, ctypes.c_float, vp, sz, vp]
    L.asd_kv_attend_shared_workspace.argtypes = [vp, vp, vp]
    L.asd_kv_attend_shared.argtypes = [vp, vp, vp, vp, i64, vp, i64, ctypes.c_float, vp, sz, vp]
    return L


def run(lib, heads, kv_heads, h, dtype, kv, start, lens, n_rows, max_new, cap, window=None, sinks=0, groups=None, only=False):
    """A call; its counts.  window and sinks, or groups: (group_start, shared_len).  only: of each launch some workgroups, to count their steps."""
    n_seqs = len(lens)
    keep = [np.array(x, np.int32) for x in (start, lens, *(groups or ()))]
    status, P = np.zeros(1, np.int32), 1 << 20
    s = asd.KvShape(heads, kv_heads, h, 64, dtype, kv)
    b = asd.KvBatch(P, P, keep[0].ctypes.data, keep[1].ctypes.data, status.ctypes.data, 4, (cap + 63) // 64, n_seqs, n_rows, max_new, cap)
    if groups:
        name, form = "shared", (ctypes.byref(asd.KvGroups(keep[2].ctypes.data, keep[3].ctypes.data, len(groups[1]))),)
    else:
        name, form = "window", (window, sinks)
    size = getattr(lib, f"asd_kv_attend_{name}_workspace")(ctypes.byref(s), ctypes.byref(b), *form)
    assert size == getattr(asd._kv_lib(), f"asd_kv_attend_{name}_workspace")(ctypes.addressof(s), ctypes.addressof(b), *(form if name == "window" else (ctypes.addressof(form[0]._obj),)))
    room = np.full(size + 2 * GUARD + 256, 0xA5, np.uint8)
    at = (-room.ctypes.data) % 256 + GUARD
    at -= (room.ctypes.data + at) % 256
    lib.cpu_begin(room.ctypes.data + at, size, n_rows, heads, kv_heads, only)
    assert getattr(lib, f"asd_kv_attend_{name}")(ctypes.byref(s), ctypes.byref(b), *form, P, heads * h, P, heads * h, 0.125, room.ctypes.data + at, size, None) == 0
    what = (start, lens, n_rows, max_new, cap, heads, kv_heads, window, sinks, groups)
    assert lib.cpu_fault() == b"", (lib.cpu_fault(), what)
    assert (room[:at] == 0xA5).all() and (room[at + size:] == 0xA5).all(), what
    if not only:
        got = np.ctypeslib.as_array((ctypes.c_uint8 * (n_rows * heads)).from_address(lib.cpu_answered())).reshape(n_rows, heads)
        want = np.zeros(n_rows, np.uint8)
        for r0, n, _, _ in mended(start, lens, n_rows, max_new, cap):
            want[r0:r0 + n] += 1
        assert (got == want[:, None]).all(), what
    own = np.ctypeslib.as_array((ctypes.c_int32 * n_seqs).from_address(lib.cpu_lows(n_seqs)))
    lows = {i: int(x) for i, x in enumerate(own) if x >= 0}
    counts = np.zeros(9, np.int64)
    lib.cpu_counts(counts.ctypes.data)
    return dict(zip(("items", "cut", "tile", "joined", "longest", "exchanges", "first", "second", "apart"), counts.tolist()), status=int(status[0]), lows=lows)


def rows_start(news):
    return [0, *np.cumsum(news).tolist()]


SHAPES = [(4, 4, 64, asd.DT_BF16, asd.DT_FP8), (16, 2, 128, asd.DT_BF16, asd.DT_BF16), (6, 2, 32, asd.DT_F32, asd.DT_F32), (8, 1, 64, asd.DT_F32, asd.DT_FP8)]


def some_arrays(r):
    """Arrays in order, or with anything in them."""
    n_seqs = r.choice([1, r.randint(1, 6), r.randint(1, 30), r.randint(60, 150)])
    cap = r.choice([64, 500, 6000, 20000])
    news = [r.choice([0, 1, 1, r.randint(1, 5), r.randint(1, 40)]) for _ in range(n_seqs)]
    lens = [min(cap, n + r.choice([0, r.randint(0, 100), r.randint(0, cap)])) for n in news]
    news = [min(a, b) for a, b in zip(news, lens)]
    start, n_rows = rows_start(news), max(1, sum(news) + r.choice([0, 0, 3]))
    max_new = max(1, max(news))
    if r.random() < 0.4:
        for _ in range(r.randint(1, 4)):
            r.choice((start, lens))[r.randrange(n_seqs)] = r.choice([-5, 0, n_rows + 2, cap + 9, r.randint(0, n_rows), 2 ** 31 - 1, -2 ** 31])
        max_new = r.randint(1, max_new)
    return start, lens, n_rows, max_new, cap


def some_groups(r, n_seqs, cap, most=150):
    n = r.choice([1, r.randint(1, 4), r.randint(1, n_seqs), r.randint(1, most)])
    start = sorted(r.randint(0, n_seqs) for _ in range(n + 1))
    if r.random() < 0.3:
        start[r.randrange(n + 1)] = r.choice([-3, n_seqs + 1, r.randint(0, n_seqs), 2 ** 31 - 1, -2 ** 31])
    return start, [r.choice([0, 1, 64, r.randint(0, 300), r.randint(0, cap), cap, cap + 5, -2]) for _ in range(n)]


@pytest.mark.parametrize("shape", SHAPES)
def test_windows(lib, shape):
    r, seen = random.Random(1), set()
    for _ in range(12):
        c = run(lib, *shape, *some_arrays(r), window=r.choice([1, 64, 300, 5000, 2 ** 31 - 1]), sinks=r.choice([0, 4, 200, 2 ** 31 - 1]))
        seen.add(c["cut"] > 0)
    assert seen == {False, True}


@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
@pytest.mark.parametrize("shape", SHAPES)
def test_shared_beginnings(lib, shape, wide):
    """wide: room for long sequences, for which the shared keys are read apart from the own ones."""
    r, n, cut = random.Random(2), 0, 0
    while n < 8:
        start, lens, n_rows, max_new, cap = some_arrays(r)
        groups = some_groups(r, len(lens), cap)
        if wide and (len(groups[1]) > len(lens) // 2 or n_rows * shape[0] // shape[1] > 64 * len(lens)):
            continue
        c = run(lib, *shape, start, lens, n_rows, max_new, 2 ** 24 if wide else cap, groups=groups)
        assert (c["joined"] > 0) or not wide
        n += 1
        cut += c["cut"] > 0
    assert cut


@pytest.mark.parametrize("form", ["window", "shared"])
@pytest.mark.parametrize("kv_heads,news,lens", [(40, [300, 1, 90, 130], [9000, 40, 90, 2100]), (40, [700, 3, 1000], [700, 3, 6000]), (64, [50, 0] + [130] * 4, [50, 5, 131, 700, 130, 2000]),
                                                (40, [64, 64], [3000, 64]), (40, [2000], [6000])])
def test_the_last_round_of_many_rows(lib, form, kv_heads, news, lens):
    """Tiles of 128 rows, of which only those that do not fill a round are cut; in order, and with arrays that are not."""
    shape = (kv_heads, kv_heads, 64, asd.DT_BF16, asd.DT_FP8)
    n_rows, cap = sum(news), 9000
    start, cut, tiles = rows_start(news), 0, set()
    for bad in ({}, {"start": (len(news) // 2, n_rows)}, {"lens": (0, 10 ** 6)}, {"start": (1, -4)}):
        a = {"start": list(start), "lens": list(lens)}
        for k, (i, x) in bad.items():
            a[k][i] = x
        kw = dict(window=3000, sinks=70) if form == "window" else dict(groups=([0, (len(news) + 1) // 2, len(news)], [60, 40]))
        c = run(lib, *shape, a["start"], a["lens"], n_rows, max(news), cap, **kw)
        tiles.add(c["tile"])
        cut += c["cut"] > 0
    assert cut and 128 in tiles and tiles <= {0, 128}


@pytest.mark.parametrize("apart", [False, True], ids=["both", "apart"])
def test_look_ups_grow_with_the_batch(lib, apart):
    """The exchanges between lanes that the longest wave takes part in are in step with sequences + groups, up to the most that a call may have.  It walks all sequences, with all groups, three
    times at most (length of a run, its item, the blocks in front), and all groups twice more (runs of the shared keys, its group's place); for 64 of either it takes 45 exchanges at most:
    11 to match them, 16 for the order of groups, 18 for a sum and a search."""
    for n, n_groups in ((4096, 2048 if apart else 4096), (8192, 4096 if apart else 8192), (65536, 32768 if apart else 65536)):
        c = run(lib, 1, 1, 32, asd.DT_BF16, asd.DT_FP8, list(range(n + 1)), [300] * n, n, 1, 600 if apart else 300, groups=([n * g // n_groups for g in range(n_groups + 1)], [100] * n_groups), only=True)
        assert (c["apart"] > 0) == apart
        assert c["longest"] <= 5 * 45 * (n // 64 + n_groups // 64) + 200, (n, n_groups)


@pytest.mark.parametrize("apart", [False, True], ids=["both", "apart"])
@pytest.mark.parametrize("kind", ["long ones at the end of sixty-four", "empty ones", "one for all", "sixty-fours"])
def test_groups_over_the_borders_of_what_a_wave_looks_at(lib, kind, apart):
    n = 400
    start = {"long ones at the end of sixty-four": [*range(64), 300, *range(300, 363), 400], "empty ones": [0] * 100 + [5] * 70 + [130] * 130 + [n], "one for all": [0, n],
             "sixty-fours": list(range(0, n, 64)) + [n]}[kind]
    r = random.Random(4)
    lens = [r.randint(200, 500) for _ in range(n)]
    shared = [r.choice([64, 100, 150]) for _ in start[1:]]
    c = run(lib, 2, 1, 32, asd.DT_BF16, asd.DT_FP8, list(range(n + 1)), lens, n, 1, 2 ** 24 if apart and len(shared) <= n // 2 else 500, groups=(start, shared))
    assert c["joined"] or not apart or len(shared) > n // 2
    # each sequence's own keys begin where its group's shared ones end
    low = dict.fromkeys(range(n), 0)
    for f0, f1, s in zip(start, start[1:], shared):
        low.update(dict.fromkeys(range(f0, f1), s))
    assert c["lows"] == low
