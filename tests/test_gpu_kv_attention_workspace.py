"""One workspace of the size for the most rows, sequences and keys, used for fewer of each too: the results of calls with their own, and nothing behind it
written."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2603_18489_amd as ec
from paper_2603_18489_amd import binding
from tests.test_gpu_kv_attention import Batch, ints

pytestmark = pytest.mark.gpu
GUARD = 4096


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("counts,lengths,heads,kv_heads,prefix,fewer", [
    ([1800], [4000], 28, 4, 0, [([1800], 4000), ([1400], 4000), ([1100], 3000), ([13], 4000), ([2], 1025), ([1], 4000)]),
    ([200] * 6, [1500] * 6, 4, 4, 700, [([200] * 6, 1500), ([61] * 6, 1500), ([200], 1500), ([3, 3], 800), ([1] * 5, 90)]),
    ([40] * 30, [600] * 30, 8, 1, 0, [([40] * 30, 600), ([11] * 17, 600), ([40, 2], 500), ([1], 300)])], ids=str)
def test_one_for_the_most_serves_fewer(counts, lengths, heads, kv_heads, prefix, fewer, cache):
    lib = ec.load_library()
    b = Batch(counts, lengths, heads, kv_heads, 128, 64, cache, prefix)
    table, shared = ints(b.table), ints(b.prefix)
    struct = binding._cache_struct(torch, b.cache)

    def cfg(rows, seqs, max_rows, keys):
        return binding.ec_kv_attention_cfg(rows, heads, seqs, max_rows, keys, b.width, len(b.prefix), prefix, 0, 0.09, b.width)
    size = lib.ec_kv_attention_workspace_bytes(C.byref(struct), C.byref(cfg(sum(counts), len(counts), max(counts), max(lengths))))
    ws = torch.full((size + GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
    for some, keys in fewer:
        rows, seqs = sum(some), len(some)
        starts, least = ints(np.cumsum([0] + some)), ints([keys] * seqs)
        out = torch.empty((rows, heads, 128), dtype=torch.bfloat16, device="cuda")
        rc = lib.ec_kv_attention(C.byref(struct), C.byref(cfg(rows, seqs, max(some), keys)), b.q.data_ptr(), heads * 128, 128, table.data_ptr(), least.data_ptr(),
                                 starts.data_ptr(), shared.data_ptr() if prefix else None, out.data_ptr(), heads * 128, 128, ws.data_ptr(), size,
                                 torch.cuda.current_stream().cuda_stream)
        assert rc == ec.EC_OK, (some, lib.ec_last_error(None))
        more = dict(prefix=shared, prefix_len=prefix) if prefix else {}
        want = ec.kv_attention(b.q[:rows], b.cache, table[:seqs], least, starts, max(some), keys, scale=0.09, **more)
        assert torch.equal(out, want)
        assert (ws[size:] == 0xA5).all()
