"""One workspace of the size for the most rows, used for fewer too: results of the calls with their own, and nothing behind it written."""
import pytest
import torch

import paper_2603_18489_amd as ec
from paper_2603_18489_amd import binding

pytestmark = pytest.mark.gpu
GUARD = 4096


def workspace(size):
    return torch.full((size + GUARD,), 0xA5, dtype=torch.uint8, device="cuda")


def stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("filters", [dict(), dict(top_p=0.9), dict(top_k=50, min_p=0.01)], ids=str)
@pytest.mark.parametrize("V,most,rows", [(126464, 34, (34, 33, 17, 16, 1)), (4097, 600, (600, 513, 512, 256, 3)), (17001, 1100, (1100, 1030, 205, 102, 1))])
def test_sampling(V, most, rows, filters):
    lib = ec.load_library()
    size = lib.ec_row_sample_workspace_bytes(most, V)
    z, u = torch.randn((most, V), device="cuda") * 3, torch.rand(most, device="cuda")
    ws = workspace(size)
    cfg = binding.ec_sample_cfg(1.0, filters.get("top_k", 0), filters.get("top_p", 1.0), filters.get("min_p", 0.0))
    for n in rows:
        tokens, stats = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty((n, 4), device="cuda")
        assert lib.ec_row_sample(z.data_ptr(), ec.EC_T_F32, n, V, V, u.data_ptr(), cfg, tokens.data_ptr(), stats.data_ptr(), ws.data_ptr(),
                                 size, stream()) == ec.EC_OK
        want = ec.row_sample(z[:n], u[:n], **filters)
        assert torch.equal(tokens, want[0]) and torch.equal(stats, want[1])
        assert (ws[size:] == 0xA5).all()


@pytest.mark.parametrize("act", ["bf16", "mxfp4"])
@pytest.mark.parametrize("n,k", [(512, 4096), (1111, 2080), (2048, 4096), (33, 12288), (130, 1504)])
def test_products(n, k, act):
    lib = ec.load_library()
    most = 1040
    x_type = ec.EC_T_MXFP4 if act == "mxfp4" else ec.EC_T_BF16
    size = lib.ec_mx_linear_workspace_bytes(x_type, most, n, k)
    assert size > 0
    packed = ec.mxfp4_pack(ec.mxfp4_quantize(torch.randn((n, k), device="cuda")))
    x = torch.randn((most, k), device="cuda").bfloat16()
    ws = workspace(size)
    for m in (most, 1024, 700, 513, 300, 130, 65, 64, 33, 17, 5, 4, 1):
        q = ec.mxfp4_quantize(x[:m])
        args = (q.codes.data_ptr(), q.scales.data_ptr()) if act == "mxfp4" else (x.data_ptr(), None)
        y = torch.empty((m, n), device="cuda")
        assert lib.ec_mx_linear(*args, x_type, m, k, packed.data.data_ptr(), n, k, y.data_ptr(), ec.EC_T_F32, n, ws.data_ptr(), size,
                                stream()) == ec.EC_OK
        assert torch.equal(y, ec.mxfp4_linear(q if act == "mxfp4" else x[:m], packed, torch.float32))
        assert (ws[size:] == 0xA5).all()
