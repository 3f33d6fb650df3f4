"""One long conversation among short ones and a chunk of a prompt: its keys are cut into runs."""
import ctypes

import pytest

import paper_2410_01028_amd as asd


def workspace(heads, kv_heads, h, n_seqs, n_rows, max_new, max_len):
    s = asd.KvShape(heads, kv_heads, h, 64, asd.DT_BF16, asd.DT_FP8)
    b = asd.KvBatch(1 << 20, 1 << 20, 1 << 20, 1 << 20, None, 4, (max_len + 63) // 64, n_seqs, n_rows, max_new, max_len)
    return asd._kv_lib().asd_kv_attend_workspace(ctypes.addressof(s), ctypes.addressof(b))


def test_tiles_of_few_rows_do_not_fill_the_card():
    """A workspace means that runs are possible: without one, a sequence's KV head is one workgroup's work from its first key to its last."""
    assert workspace(64, 8, 128, 130, 641, 512, 60000) > 0         # 128 short ones, a long one, a chunk
    assert workspace(64, 8, 128, 2, 513, 512, 60000) > 0
    assert workspace(32, 32, 128, 4, 6901, 2048, 2048) == 0        # prompts: as many full tiles as the card takes


@pytest.mark.gpu
@pytest.mark.parametrize("kv", ["fp8", "bf16"])
def test_a_long_conversation_among_short_ones_and_a_chunk(kv):
    from test_gpu_kv_ops import Pool, check_attend
    news, total = [1] * 128 + [1, 300], [40 + 3 * i for i in range(128)] + [20000, 700]
    p = Pool("bf16", kv, 32, 8, 64, 64, list(zip(news, total)), seed=31)
    k, v = p.fill()
    b = p.batch(news, total)
    assert p.cache.attend_workspace(b) > 0
    q = p.normal(sum(news), 32, 64, scale=2.0)
    out = p.cache.attend(b, q)
    b.check()
    check_attend(p, news, total, q, out, k, v, 0.125)
