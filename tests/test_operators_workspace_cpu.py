"""Workspaces of the sampling and 4-bit entry points: one for so many rows serves fewer, wherever the blocks change."""
import pytest

import paper_2603_18489_amd as ec


@pytest.mark.parametrize("vocab", [2, 4096, 4097, 8193, 17001, 126464, 152064, 163840])
def test_sampling_workspace_grows_with_the_rows(vocab):
    lib = ec.load_library()
    sizes = [lib.ec_row_sample_workspace_bytes(rows, vocab) for rows in range(2200)] + [lib.ec_row_sample_workspace_bytes(65535, vocab)]
    assert sizes[0] == 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))
    assert (sizes[1] > 0) == (vocab > 4096)


@pytest.mark.parametrize("x_type", [ec.EC_T_BF16, ec.EC_T_MXFP4])
@pytest.mark.parametrize("n,k", [(1, 32), (44, 1504), (64, 18944), (1000, 2048), (4096, 4096), (4096, 12288), (24576, 4096), (99001, 4096),
                                 (126464, 4096), (2 ** 20, 131072)])
def test_product_workspace_grows_with_the_rows(n, k, x_type):
    lib = ec.load_library()
    sizes = [lib.ec_mx_linear_workspace_bytes(x_type, rows, n, k) for rows in list(range(2100)) + [2 ** 19]]
    assert sizes[0] == 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))
