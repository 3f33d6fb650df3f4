"""Batches whose arrays say what cannot be: rows that several sequences claim."""
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


# heads, KV heads, head dim, cache type, row_start, lengths, rows, most new rows
CLAIMS = {"tiles of 128 rows, long and short": (64, 8, 128, "fp8", [64 * (i % 2) for i in range(129)], [8192] + [64] * 125 + [8192, 64], 64, 64),
          "tiles of 128 rows, one length": (128, 16, 128, "bf16", [100 * (i % 2) for i in range(6)], [1536] * 5, 100, 100),
          "tiles of 16 rows": (32, 32, 64, "fp8", [9 * (i % 2) for i in range(41)], [3000] * 40, 9, 9),
          "behind the first 64": (8, 2, 64, "bf16", [*range(70), 5, 75, 60, 80, 85], [200 + i for i in range(74)], 90, 20)}


@pytest.mark.parametrize("kind", list(CLAIMS))
def test_rows_that_several_sequences_claim(kind):
    """The first one has them; nothing is written outside the workspace, to rows that none has, or to pages of sequences without rows."""
    heads, kv_heads, h, kv, start, lens, n_rows, max_new = CLAIMS[kind]
    p = Pool("bf16", kv, heads, kv_heads, h, 64, [(0, n) for n in lens], seed=21)
    k, v = p.fill()
    claimed = rows_of(start, n_rows, max_new)
    having = [i for i, (_, n) in enumerate(claimed) if n]
    assert 0 < len(having) < len(lens)
    b = batch(p, start, lens, n_rows, max_new)
    q, new_k, new_v = p.normal(n_rows, heads, h), p.normal(n_rows, kv_heads, h), p.normal(n_rows, kv_heads, h)
    need = p.cache.attend_workspace(b)
    buffer = torch.full((need + (16 << 20),), 0xA5, dtype=torch.uint8, device=DEV)
    out = torch.full((n_rows, heads, h), 7.0, dtype=torch.bfloat16, device=DEV)
    p.cache.attend(b, q, out=out, workspace=buffer[8 << 20:][:need])
    with pytest.raises(asd.AsdError, match="rows or lengths"):
        b.check()
    assert bool((buffer[:8 << 20] == 0xA5).all()) and bool((buffer[(8 << 20) + need:] == 0xA5).all())
    free = torch.ones(n_rows, dtype=torch.bool, device=DEV)
    for i in having:
        r0, n = claimed[i]
        check_attend(p, [n], [lens[i]], q[r0:r0 + n], out[r0:r0 + n], k[i:i + 1], v[i:i + 1], h ** -0.5)
        free[r0:r0 + n] = False
    assert bool((out[free] == 7.0).all())
    before = p.pages.clone()
    turned = p.cache.append(b, q, new_k, new_v, q_out=torch.full_like(q, 7.0))
    got = p.cache.read(b, torch.full_like(new_k, 7.0), torch.full_like(new_v, 7.0))
    with pytest.raises(asd.AsdError, match="rows or lengths"):
        b.check()
    assert bool((turned[free] == 7.0).all()) and torch.equal(turned[~free], q[~free])
    for x, new in zip(got, (new_k, new_v)):
        assert bool((x[free] == 7.0).all())
        # (8 bits: half a step, 2^-4 of the value, or of 2^-6 times the scale's unit at most max|x| / 224, and the rounding to bf16)
        slack = (new.double().abs() * 2.0 ** -4 + new.double().abs().amax(-1, keepdim=True) * 2.0 ** -10 / 224) if kv == "fp8" else torch.zeros_like(new).double()
        assert bool(((x.double() - new.double()).abs() <= slack)[~free].all())
    none = [i for i in range(len(lens)) if i not in having]
    rest = p.table[none].flatten().long().to(DEV)
    assert torch.equal(p.pages[rest], before[rest])
