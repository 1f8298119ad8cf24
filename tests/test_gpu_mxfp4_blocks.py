"""Products in 4 bits of more than 64 rows, by every block that their sizes can get: ragged rows, features and ends of K, K in ranges, scales
that have to be laid out first.  Bounds as derived in tests/test_gpu_mxfp4.py."""
import pytest
import torch

import paper_2603_18489_amd as ec

BF16, MX = ec.EC_T_BF16, ec.EC_T_MXFP4
# type of the rows; rows, features, k; block rows, block features, ranges of K
CASES = [
    (BF16, 73, 269, 288, (64, 256, 1)), (BF16, 79, 258, 1120, (64, 256, 2)), (BF16, 73, 262, 2144, (64, 256, 4)),
    (BF16, 4339, 777, 288, (128, 128, 1)), (BF16, 581, 3094, 2592, (128, 128, 2)), (BF16, 773, 1095, 2368, (128, 128, 4)),
    (BF16, 143, 22570, 288, (128, 256, 1)), (BF16, 70, 16761, 4928, (128, 256, 2)), (BF16, 263, 3175, 2336, (128, 256, 4)),
    (MX, 71, 283, 288, (64, 256, 1)), (MX, 85, 258, 2368, (64, 256, 2)), (MX, 69, 261, 3872, (64, 256, 4)),
    (MX, 4233, 787, 288, (128, 128, 1)), (MX, 600, 3135, 5024, (128, 128, 2)), (MX, 329, 2609, 3936, (128, 128, 4)),
    (MX, 145, 23954, 288, (128, 256, 1)), (MX, 69, 33551, 32, (128, 256, 1)), (MX, 70, 17134, 8448, (128, 256, 2)), (MX, 135, 5498, 4896, (128, 256, 4)),
    (MX, 283, 22962, 288, (192, 256, 1)), (MX, 131, 24755, 9952, (192, 256, 2)), (MX, 130, 11081, 7296, (192, 256, 4)),
    (MX, 257, 38739, 288, (192, 384, 1)), (MX, 69, 66490, 160, (192, 384, 1)), (MX, 139, 33127, 9088, (192, 384, 2)), (MX, 131, 23626, 8000, (192, 384, 4)),
    (MX, 385, 25150, 288, (256, 256, 1)), (MX, 3001, 8204, 1056, (256, 256, 1)), (MX, 4100, 4100, 4192, (192, 384, 1)), (MX, 2049, 4100, 1056, (192, 256, 1)), (MX, 194, 8825, 13280, (256, 256, 4)),
]


@pytest.mark.parametrize("kind,m,n,k,shape", CASES)
def test_the_sizes_get_these_blocks(kind, m, n, k, shape):
    """(without a GPU: so that a rule that changes does not take a block out of the tests below)"""
    assert ec.mx_blocks(kind, m, n, k) == shape


def test_what_the_query_refuses():
    lib = ec.load_library()
    for args in ((ec.EC_T_F32, 4, 20, 64), (BF16, 0, 20, 64), (BF16, 2 ** 19 + 1, 20, 64), (MX, 4, 0, 64), (MX, 4, 20, 40)):
        with pytest.raises(ec.EcError):
            ec.mx_blocks(*args)
    assert lib.ec_debug_mx_blocks(BF16, 4, 20, 64, None) == ec.EC_ERR_ARG
    assert ec.mx_blocks(BF16, 17, 20, 64)[0] == 32


@pytest.mark.gpu
@pytest.mark.parametrize("kind,m,n,k,shape", CASES)
def test_against_64_bits(kind, m, n, k, shape):
    """Results in both types, in rows with room behind them that is left alone; scales at every alignment, some blocks of no value."""
    lib = ec.load_library()
    gen = torch.Generator(device="cuda").manual_seed(m * n + k)
    pick = lambda lo, hi, size: torch.randint(lo, hi, size, dtype=torch.uint8, device="cuda", generator=gen)
    w = ec.Mxfp4(pick(0, 256, (n, k // 2)), pick(120, 131, (n, k // 32)))
    w.codes[n // 2] = 0
    packed = ec.mxfp4_pack(w)
    wv = ec.mxfp4_dequantize(w).double()
    if kind == MX:
        q = ec.Mxfp4(pick(0, 256, (m, k // 2)), pick(122, 133, (m, k // 32)))
        q.scales[m - 1, k // 32 - 1] = 255            # NaN: the last row has no values
        q.codes[0] = 0
        room = torch.empty(q.scales.numel() + 1, dtype=torch.uint8, device="cuda")
        moved = room[1:].view_as(q.scales).copy_(q.scales)
        xv, rows, ld = ec.mxfp4_dequantize(q).double(), [(q.codes, s) for s in (q.scales, moved)], k
    else:
        buf = torch.randn((m, k + 8), device="cuda", generator=gen).bfloat16()
        buf[m - 1, k - 1] = float("nan")
        buf[:, k:] = float("nan")
        buf[0] = 0
        xv, rows, ld = buf[:, :k].double(), [(buf, None)], k + 8
    want, size = xv @ wv.t().contiguous(), xv.abs() @ wv.abs().t().contiguous()
    assert want[m - 1].isnan().all()
    bound = (k / 32 + 144) * 2.0 ** -23 * size[:m - 1]
    need = lib.ec_mx_linear_workspace_bytes(kind, m, n, k)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    for dtype, y_kind in ((torch.float32, ec.EC_T_F32), (torch.bfloat16, ec.EC_T_BF16)):
        for gap in (0, 8 - n % 8, 3):
            for x, scales in rows:
                y = torch.full((m + 2, n + gap), 77.0, dtype=dtype, device="cuda")
                assert lib.ec_mx_linear(x.data_ptr(), scales.data_ptr() if scales is not None else None, kind, m, ld, packed.data.data_ptr(), n, k,
                                        y.data_ptr(), y_kind, n + gap, ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == ec.EC_OK
                assert (y[m:] == 77).all() and (y[:, n:] == 77).all()
                assert y[m - 1, :n].isnan().all() and (y[0, :n] == 0).all() and (y[:m - 1, n // 2] == 0).all()
                off = (y[:m - 1, :n].double() - want[:m - 1]).abs()
                assert (off <= bound + (2.0 ** -8 * want[:m - 1].abs() if dtype == torch.bfloat16 else 0)).all()
