"""Tensors of no rows, whose strides may be anything: numpy gives its empty arrays zeros, which torch keeps."""
import numpy as np
import pytest
import torch

import paper_2603_18489_amd as ec
from paper_2603_18489_amd import binding


def test_strides_of_no_rows_do_not_count():
    none = torch.from_numpy(np.ones((0, 2, 64), dtype=np.float32))
    other = torch.empty((2, 64, 0)).permute(2, 0, 1)
    for x in (none, other):
        assert x.stride(2) != 1 or x.stride(0) == 1
        assert binding._heads_of(x, "x") == (0, 2, 64, 0, x.stride(1))
    with pytest.raises(ValueError, match="next to each other"):
        binding._heads_of(torch.ones((1, 2, 128))[..., ::2], "x")
    # (all that is left to refuse is where they are)
    cache, plan = ec.kv_cache(3, 2, 64, 32, device="cpu"), ec.RotaryPlan(torch.zeros(32, dtype=torch.float64), 64, False, 1.0)
    at, table, lengths = torch.zeros(0, dtype=torch.int32), torch.zeros((1, 1), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for call in (lambda: ec.rotary(none, at, plan), lambda: ec.kv_write(cache, none, none, at),
                 lambda: ec.kv_attention(none.bfloat16(), cache, table, lengths)):
        with pytest.raises(ValueError, match="GPU"):
            call()
