"""What mxfp4_linear refuses as its matrix, before it looks for a GPU: the kernels read it by bytes, one after the other."""
import pytest
import torch

import paper_2603_18489_amd as ec


@pytest.mark.parametrize("data", [torch.zeros(4352, dtype=torch.int8), torch.zeros(4352, dtype=torch.float32), torch.zeros(4352, dtype=torch.bool),
                                  torch.zeros(2 * 4352, dtype=torch.uint8)[::2], torch.zeros(1, dtype=torch.uint8).expand(4352),
                                  torch.zeros((64, 68), dtype=torch.uint8).t()],
                         ids=["int8", "float32", "bool", "every other byte", "one byte", "transposed"])
def test_a_matrix_of_another_type_or_order(data):
    w = ec.Mxfp4Matrix(data, 20, 64)
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    q = ec.Mxfp4(torch.zeros((4, 32), dtype=torch.uint8), torch.zeros((4, 2), dtype=torch.uint8))
    for rows in (x, q):
        with pytest.raises(ValueError, match="mxfp4_pack"):
            ec.mxfp4_linear(rows, w)
    with pytest.raises(ValueError, match="GPU"):
        ec.mxfp4_linear(x, ec.Mxfp4Matrix(torch.zeros(4352, dtype=torch.uint8), 20, 64))
