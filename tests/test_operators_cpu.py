"""Refusals of the sampling and 4-bit entry points, which happen before anything touches a GPU."""
import ctypes as C

import pytest
import torch

import paper_2603_18489_amd as ec
from paper_2603_18489_amd import binding

P = 1 << 20          # addresses that nothing reads: every call here is refused, or has no rows
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    return ec.load_library()


def sample(lib, logits=P, type=0, rows=4, vocab=100, ld=100, uniforms=P, cfg=(1.0, 0, 1.0, 0.0), tokens=P, stats=P, ws=P, size=None):
    size = lib.ec_row_sample_workspace_bytes(rows, vocab) if size is None else size
    return lib.ec_row_sample(logits, type, rows, vocab, ld, uniforms, binding.ec_sample_cfg(*cfg) if cfg else None, tokens, stats,
                             ws, size, None)


@pytest.mark.parametrize("bad", [dict(logits=None), dict(uniforms=None), dict(tokens=None), dict(stats=None), dict(cfg=None),
                                 dict(type=2), dict(type=-1), dict(rows=-1), dict(rows=65536), dict(vocab=1), dict(vocab=163841, ld=163841),
                                 dict(ld=99), dict(stats=P + 8), dict(logits=P + 2), dict(type=1, logits=P + 1), dict(tokens=P + 1),
                                 dict(uniforms=P + 2)] +
                         [dict(cfg=c) for c in ((-0.5, 0, 1.0, 0.0), (NAN, 0, 1.0, 0.0), (INF, 0, 1.0, 0.0), (1.0, -1, 1.0, 0.0),
                                                (1.0, 0, 0.0, 0.0), (1.0, 0, 1.5, 0.0), (1.0, 0, NAN, 0.0), (1.0, 0, 1.0, -0.1),
                                                (1.0, 0, 1.0, 1.1), (1.0, 0, 1.0, NAN))], ids=str)
def test_sample_refuses(lib, bad):
    assert sample(lib, **bad) == ec.EC_ERR_ARG
    assert lib.ec_last_error(None)


def test_sample_workspace(lib):
    big = dict(vocab=40000, ld=40000)
    assert sample(lib, ws=None, **big) == sample(lib, ws=P + 128, **big) == ec.EC_ERR_WORKSPACE
    need = lib.ec_row_sample_workspace_bytes(4, 40000)
    assert need > 0 and sample(lib, size=need - 1, **big) == ec.EC_ERR_WORKSPACE
    for rows, vocab in ((-1, 40000), (65536, 40000), (4, 1), (4, 163841), (4, 4096), (0, 40000)):
        assert lib.ec_row_sample_workspace_bytes(rows, vocab) == 0
    assert sample(lib, rows=0, logits=None, uniforms=None, tokens=None, stats=None, ws=None) == ec.EC_OK


def quantize(lib, x=P, type=0, rows=4, k=64, ld=64, codes=P, scales=P):
    return lib.ec_mx_quantize(x, type, rows, k, ld, codes, scales, None)


def dequantize(lib, x=P, type=0, rows=4, k=64, ld=64, codes=P, scales=P):
    return lib.ec_mx_dequantize(codes, scales, rows, k, x, type, ld, None)


@pytest.mark.parametrize("call", [quantize, dequantize])
@pytest.mark.parametrize("bad", [dict(x=None), dict(codes=None), dict(scales=None), dict(type=2), dict(type=-1), dict(rows=-1),
                                 dict(rows=2 ** 24 + 1), dict(k=0), dict(k=-32), dict(k=48), dict(k=131104, ld=131104), dict(ld=63),
                                 dict(codes=P + 8), dict(x=P + 2), dict(type=1, x=P + 1)], ids=str)
def test_to_and_from_refuse(lib, call, bad):
    assert call(lib, **bad) == ec.EC_ERR_ARG
    assert lib.ec_last_error(None)


def test_to_and_from_without_rows(lib):
    assert quantize(lib, rows=0, x=None, codes=None, scales=None) == ec.EC_OK
    assert dequantize(lib, rows=0, x=None, codes=None, scales=None) == ec.EC_OK


def pack(lib, codes=P, scales=P, n=20, k=64, packed=P, size=1 << 30):
    return lib.ec_mx_pack(codes, scales, n, k, packed, size, None)


def linear(lib, x=P, x_scales=P, x_type=1, rows=4, ld=64, packed=P, n=20, k=64, y=P, y_type=0, ldy=20, ws=P, size=1 << 30):
    return lib.ec_mx_linear(x, x_scales, x_type, rows, ld, packed, n, k, y, y_type, ldy, ws, size, None)


@pytest.mark.parametrize("bad", [dict(codes=None), dict(scales=None), dict(n=0), dict(n=2 ** 20 + 1), dict(k=0), dict(k=33),
                                 dict(k=131104), dict(codes=P + 4)], ids=str)
def test_pack_refuses(lib, bad):
    assert pack(lib, **bad) == ec.EC_ERR_ARG
    assert pack(lib, packed=None) == pack(lib, packed=P + 64) == ec.EC_ERR_WORKSPACE
    assert pack(lib, size=lib.ec_mx_packed_bytes(20, 64) - 1) == ec.EC_ERR_WORKSPACE
    if "n" in bad or "k" in bad:
        assert lib.ec_mx_packed_bytes(bad.get("n", 20), bad.get("k", 64)) == 0


def test_packed_bytes_hold_the_matrix(lib):
    for n, k in ((1, 32), (16, 128), (17, 160), (24576, 4096), (2 ** 20, 131072)):
        assert lib.ec_mx_packed_bytes(n, k) >= n * k * 17 // 32


@pytest.mark.parametrize("bad", [dict(x=None), dict(packed=None), dict(y=None), dict(x_type=0), dict(x_type=3), dict(y_type=2),
                                 dict(rows=-1), dict(rows=2 ** 19 + 1), dict(n=0), dict(n=2 ** 20 + 1, ldy=2 ** 21), dict(k=0), dict(k=40),
                                 dict(k=131104, ld=131104), dict(ld=56), dict(ld=68), dict(ldy=19), dict(x=P + 8), dict(packed=P + 64),
                                 dict(y=P + 2), dict(y=P + 1, y_type=1), dict(x_type=2, x_scales=None)], ids=str)
def test_linear_refuses(lib, bad):
    assert linear(lib, **bad) == ec.EC_ERR_ARG
    assert lib.ec_last_error(None)


def test_linear_workspace(lib):
    for x_type, rows, n, k in ((1, 34, 4096, 12288), (2, 34, 4096, 12288), (1, 128, 4096, 4096), (2, 128, 4096, 4096), (2, 2 ** 19, 1000, 64)):
        need = lib.ec_mx_linear_workspace_bytes(x_type, rows, n, k)
        size = dict(x_type=x_type, rows=rows, n=n, k=k, ld=k, ldy=n)
        assert need > 0
        assert linear(lib, size=need - 1, **size) == linear(lib, ws=None, **size) == linear(lib, ws=P + 16, **size) == ec.EC_ERR_WORKSPACE
    for args in ((0, 4, 20, 64), (1, -1, 20, 64), (1, 2 ** 19 + 1, 20, 64), (1, 4, 0, 64), (1, 4, 20, 40)):
        assert lib.ec_mx_linear_workspace_bytes(*args) == 0
    assert linear(lib, rows=0, x=None, packed=None, y=None, ws=None) == ec.EC_OK


def test_the_binding_refuses_what_is_not_on_a_gpu_or_has_another_form():
    z, u = torch.zeros((4, 100)), torch.zeros(4)
    q = ec.Mxfp4(torch.zeros((20, 32), dtype=torch.uint8), torch.zeros((20, 2), dtype=torch.uint8))
    w = ec.Mxfp4Matrix(torch.zeros(4096, dtype=torch.uint8), 20, 64)
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    for call in (lambda: ec.row_sample(z, u), lambda: ec.mxfp4_quantize(z[:, :96]), lambda: ec.mxfp4_dequantize(q), lambda: ec.mxfp4_pack(q),
                 lambda: ec.mxfp4_linear(x, w), lambda: ec.mxfp4_linear(q, w)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    for call in (lambda: ec.row_sample(z.half(), u), lambda: ec.row_sample(z[0], u), lambda: ec.row_sample(z.t(), u),
                 lambda: ec.row_sample(z, u[:3]), lambda: ec.row_sample(z, u.double()), lambda: ec.row_sample(z, torch.zeros(8)[::2]),
                 lambda: ec.row_sample(z[:1].expand(4, 100), u),
                 lambda: ec.mxfp4_quantize(z.half()), lambda: ec.mxfp4_dequantize(q, torch.float16),
                 lambda: ec.mxfp4_pack(ec.Mxfp4(q.codes, q.scales[:, :1])), lambda: ec.mxfp4_pack(ec.Mxfp4(q.codes[::2], q.scales[::2])),
                 lambda: ec.mxfp4_linear(x.float(), w), lambda: ec.mxfp4_linear(x[:, :32], w), lambda: ec.mxfp4_linear(x, w, torch.float16)):
        with pytest.raises(ValueError):
            call()


def test_the_binding_refuses_numbers_that_its_arguments_do_not_hold():
    many, wide = torch.empty((2 ** 32 + 3, 32), device="meta"), torch.empty((3, 2 ** 32 + 32), device="meta")
    for call in (lambda: ec.mxfp4_quantize(many), lambda: ec.mxfp4_quantize(wide),
                 lambda: ec.row_sample(many, torch.empty(2 ** 32 + 3, device="meta")),
                 lambda: ec.mxfp4_dequantize(ec.Mxfp4(torch.empty((2 ** 32 + 3, 16), dtype=torch.uint8, device="meta"),
                                                      torch.empty((2 ** 32 + 3, 1), dtype=torch.uint8, device="meta")))):
        with pytest.raises(ValueError, match="2\\^31"):
            call()
