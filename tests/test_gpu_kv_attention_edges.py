"""Attention over a paged cache: batches of no sequences, starts and lengths that are none."""
import numpy as np
import pytest
import torch

import paper_2603_18489_amd as ec
from tests.test_gpu_kv_attention import Batch, ints

pytestmark = pytest.mark.gpu


def test_a_batch_of_no_sequences():
    cache = ec.kv_cache(3, 2, 64, 32)
    q = torch.randn((5, 4, 64), device="cuda").bfloat16()
    table, none = torch.zeros((0, 3), dtype=torch.int32, device="cuda"), ints([])
    assert ec.kv_attention(q[:0], cache, table, none).shape == (0, 4, 64)
    assert ec.kv_attention(q[:0], cache, table, none, ints([0])).shape == (0, 4, 64)
    assert ec.kv_attention(q[:0], cache, table, none, prefix=ints([1]), prefix_len=7).shape == (0, 4, 64)
    assert (ec.kv_attention(q, cache, table, none, ints([0])) == 0).all()       # rows of no sequence
    out = torch.full_like(q, 7.0)
    assert ec.kv_attention(q, cache, table, none, ints([0]), out=out) is out and (out == 7).all()
    for bad in (lambda: ec.kv_attention(q, cache, table, none), lambda: ec.kv_attention(q[:0], cache, table, none, max_rows=1)):
        with pytest.raises(ValueError, match="rows / seqs"):
            bad()


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("counts,most,prefix", [([6, 2, 5], 6, 33), ([6, 2, 5], 6, 0), ([40, 20, 9], 40, 0), ([150, 3, 90], 150, 700), ([1, 1, 1], 1, 3000)], ids=str)
def test_starts_and_lengths_that_are_none(counts, most, prefix, cache):
    """what is written are the rows that clamped starts name, and nothing before or behind the result: it lies in the middle of a larger one"""
    b = Batch(counts, [40, 50, 1100], 4, 2, 128, 32, cache, prefix)
    rows, far = sum(counts), 2 ** 31 - 1
    all_ = torch.empty((rows + 64, 6, 160), dtype=torch.bfloat16, device="cuda")
    out = all_[32:32 + rows, 1:5, 16:144]
    right = list(b.starts)
    for starts in (right, [0, -5, rows + 7, rows], [rows, 8, 6, 0], [-1] * 4, [far, -far - 1, 0, rows], [1, 1, 2, rows - 1], [far] * 4, [0, 0, 0, far]):
        for lengths in (b.lengths, [-1, far, -far - 1], [far] * 3):
            all_.fill_(7.0)
            more = dict(prefix=ints(b.prefix), prefix_len=prefix) if prefix else {}
            ec.kv_attention(b.q, b.cache, ints(b.table), ints(lengths), ints(starts), most, 1100, out=out, causal=lengths is b.lengths, **more)
            named = np.zeros(rows, dtype=bool)
            at = np.clip(starts, 0, rows)
            for first, end in zip(at[:-1], at[1:]):
                named[first:min(max(end, first), first + most)] = True
            got = all_.float().cpu().numpy()
            inside = got[32:32 + rows, 1:5, 16:144].copy()
            got[32:32 + rows, 1:5, 16:144] = 7
            assert (got == 7).all(), (starts, lengths)
            assert (inside[~named] == 7).all() and (inside[named] != 7).any(axis=(1, 2)).all(), (starts, lengths)


def test_no_rows_of_any_strides():
    none = torch.from_numpy(np.ones((0, 2, 64), dtype=np.float32)).cuda()
    cache, plan = ec.kv_cache(3, 2, 64, 32), ec.rotary_plan(64)
    ec.kv_write(cache, none, none, ints([]))
    assert (cache.data == 0).all()
    assert ec.rotary(none, ints([]), plan).shape == (0, 2, 64)
    assert ec.kv_attention(none.bfloat16(), cache, ints([[0]]), ints([5])).shape == (0, 2, 64)
