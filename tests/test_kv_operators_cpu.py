"""Refusals of the rotary, cache and attention entry points, which happen before anything touches a GPU, the frequencies of rotary positions, and the
layout of their structures."""
import ctypes as C
import os
import subprocess
import tempfile

import numpy as np
import pytest
import torch

import paper_2603_18489_amd as ec
from paper_2603_18489_amd import binding

P = 1 << 20          # addresses that nothing reads: every call here is refused, or has no rows
NAN, INF = float("nan"), float("inf")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    return ec.load_library()


def test_structures_match_the_header():
    prog = r'''
    #include <stdio.h>
    #include <stddef.h>
    #include "ec.h"
    int main(void) {
      printf("%zu %zu %zu %zu %zu %zu %d\n", sizeof(ec_rotary_cfg), offsetof(ec_rotary_cfg, base), sizeof(ec_kv_cache), sizeof(ec_kv_attention_cfg),
             offsetof(ec_kv_attention_cfg, scale), offsetof(ec_kv_attention_cfg, table_ld), EC_T_E4M3);
      return 0;
    }'''
    with tempfile.TemporaryDirectory() as td:
        open(os.path.join(td, "s.c"), "w").write(prog)
        subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), os.path.join(td, "s.c"), "-o", os.path.join(td, "s")])
        got = [int(v) for v in subprocess.check_output([os.path.join(td, "s")]).split()]
    assert got == [C.sizeof(ec.ec_rotary_cfg), ec.ec_rotary_cfg.base.offset, C.sizeof(ec.ec_kv_cache), C.sizeof(ec.ec_kv_attention_cfg),
                   ec.ec_kv_attention_cfg.scale.offset, ec.ec_kv_attention_cfg.table_ld.offset, ec.EC_T_E4M3]


def frequencies(lib, dim=8, base=10000.0, factor=1.0, original=0.0, low=1.0, high=4.0):
    turns = np.full(300, -1.0)
    return lib.ec_rotary_frequencies(C.byref(ec.ec_rotary_cfg(dim, base, factor, original, low, high)), turns.ctypes.data), turns


@pytest.mark.parametrize("bad", [dict(dim=0), dict(dim=-2), dict(dim=7), dict(dim=514), dict(base=0.0), dict(base=-1.0), dict(base=INF), dict(base=NAN),
                                 dict(factor=0.5), dict(factor=INF), dict(factor=NAN), dict(original=-1.0), dict(original=NAN), dict(original=INF),
                                 dict(original=10.0, low=4.0), dict(original=10.0, low=NAN), dict(original=10.0, high=INF)], ids=str)
def test_frequencies_refuse(lib, bad):
    rc, turns = frequencies(lib, **bad)
    assert rc == ec.EC_ERR_ARG and (turns == -1).all() and lib.ec_last_error(None)
    assert lib.ec_rotary_frequencies(None, turns.ctypes.data) == ec.EC_ERR_ARG
    assert lib.ec_rotary_frequencies(C.byref(ec.ec_rotary_cfg(8, 1e4, 1, 0, 1, 4)), None) == ec.EC_ERR_ARG


def test_frequencies(lib):
    theta = 500000.0 ** (-np.arange(64) / 64)
    for factor, original, low, high in ((1, 0, 1, 4), (8, 0, 1, 4), (8, 8192, 1, 4), (40, 4096, 1, 32), (1, 4096, 1, 32)):
        r = original * theta / (2 * np.pi)
        share = np.clip((r - low) / (high - low), 0, 1) if original else 0
        rc, turns = frequencies(lib, 128, 500000.0, factor, original, low, high)
        assert rc == ec.EC_OK and (turns[64:] == -1).all()
        np.testing.assert_allclose(turns[:64] * 2 * np.pi, share * theta + (1 - share) * theta / factor, rtol=1e-14)


def rotary(lib, x=P, type=0, rows=3, heads=4, head_dim=64, ld=256, ld_head=64, positions=P, turns=P, dim=64, interleaved=0, amplitude=1.0, inverse=0,
           out=2 * P, out_ld=256, out_ld_head=64):
    return lib.ec_rotary(x, type, rows, heads, head_dim, ld, ld_head, positions, turns, dim, interleaved, amplitude, inverse, out, out_ld, out_ld_head, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(positions=None), dict(turns=None), dict(out=None), dict(type=2), dict(type=3), dict(type=-1), dict(rows=-1),
                                 dict(rows=2 ** 24 + 1), dict(heads=0), dict(heads=1025), dict(head_dim=1), dict(head_dim=513), dict(dim=0), dict(dim=3),
                                 dict(dim=66), dict(amplitude=NAN), dict(amplitude=INF), dict(out_ld=255), dict(out_ld_head=63), dict(out_ld=0),
                                 dict(out=P, out_ld=512), dict(out=P, ld=512), dict(x=P + 2), dict(out=P + 1, type=1), dict(positions=P + 2),
                                 dict(turns=P + 4)], ids=str)
def test_rotary_refuses(lib, bad):
    assert rotary(lib, **bad) == ec.EC_ERR_ARG
    assert lib.ec_last_error(None)


def test_rotary_without_rows(lib):
    assert rotary(lib, rows=0, x=None, positions=None, turns=None, out=None) == ec.EC_OK


def cache(data=P, type=3, pages=10, page=64, kv_heads=4, head_dim=128):
    return ec.ec_kv_cache(data, type, pages, page, kv_heads, head_dim)


BAD_CACHES = [dict(type=0), dict(type=2), dict(type=4), dict(pages=0), dict(pages=-1), dict(pages=2 ** 25), dict(page=16), dict(page=48), dict(page=512),
              dict(page=0), dict(kv_heads=0), dict(kv_heads=1025), dict(head_dim=96), dict(head_dim=256), dict(head_dim=0)]


def test_cache_bytes(lib):
    for type, size in ((3, 1), (1, 2)):
        for pages, page, heads, hd in ((1, 32, 1, 64), (7, 256, 3, 128), (2 ** 20, 32, 8, 128)):
            need = lib.ec_kv_bytes(C.byref(cache(None, type, pages, page, heads, hd)))
            assert need == 2 * pages * page * heads * (hd * size + 1)
    for bad in BAD_CACHES:
        assert lib.ec_kv_bytes(C.byref(cache(**bad))) == 0
    assert lib.ec_kv_bytes(None) == 0


def write(lib, c=None, k=P, v=P, type=0, rows=3, k_ld=512, k_head=128, v_ld=512, v_head=128, slots=P, **more):
    c = C.byref(cache(**more)) if c is None else c
    return lib.ec_kv_write(c, k, v, type, rows, k_ld, k_head, v_ld, v_head, slots, None)


def read(lib, c=None, k=P, v=P, type=0, rows=3, k_ld=512, k_head=128, v_ld=512, v_head=128, slots=P, **more):
    c = C.byref(cache(**more)) if c is None else c
    return lib.ec_kv_read(c, slots, rows, k, v, type, k_ld, k_head, v_ld, v_head, None)


@pytest.mark.parametrize("call", [write, read])
@pytest.mark.parametrize("bad", BAD_CACHES + [dict(data=None), dict(data=P + 128), dict(k=None), dict(v=None), dict(slots=None), dict(rows=-1), dict(rows=2 ** 20 + 1),
                                              dict(type=2), dict(k=P + 2), dict(v=P + 1), dict(slots=P + 2)], ids=str)
def test_write_and_read_refuse(lib, call, bad):
    if "type" in bad and bad["type"] != 2:      # the cache's
        c = cache(**bad)
        assert (lib.ec_kv_write(C.byref(c), P, P, 0, 3, 512, 128, 512, 128, P, None) if call is write else
                lib.ec_kv_read(C.byref(c), P, 3, P, P, 0, 512, 128, 512, 128, None)) == ec.EC_ERR_ARG
    else:
        assert call(lib, **bad) == ec.EC_ERR_ARG
    assert lib.ec_last_error(None)


def test_write_and_read_edges(lib):
    for call in (write, read):
        assert call(lib, rows=0, k=None, v=None, slots=None, data=None) == ec.EC_OK
    assert lib.ec_kv_write(None, P, P, 0, 3, 512, 128, 512, 128, P, None) == ec.EC_ERR_ARG
    assert read(lib, k_ld=511) == read(lib, v_ld=0) == read(lib, v_head=127) == ec.EC_ERR_ARG


def attention(lib, c=None, q=P, ld=1024, ld_head=128, table=P, lengths=P, starts=P, prefix=P, out=2 * P, out_ld=1024, out_ld_head=128, ws=P, size=1 << 40,
              rows=12, heads=8, seqs=3, max_rows=12, max_keys=500, table_pages=9, prefix_pages=5, prefix_len=300, causal=0, scale=0.1, table_ld=9, **more):
    cfg = ec.ec_kv_attention_cfg(rows, heads, seqs, max_rows, max_keys, table_pages, prefix_pages, prefix_len, causal, scale, table_ld)
    c = cache(**more) if c is None else c
    assert lib.ec_kv_attention_workspace_bytes(C.byref(c), C.byref(cfg)) >= 0
    return lib.ec_kv_attention(C.byref(c), C.byref(cfg), q, ld, ld_head, table, lengths, starts, prefix, out, out_ld, out_ld_head, ws, size, None)


@pytest.mark.parametrize("bad", BAD_CACHES + [dict(data=None), dict(data=P + 64), dict(q=None), dict(out=None), dict(lengths=None), dict(table=None), dict(prefix=None),
                                              dict(starts=None), dict(q=P + 8), dict(out=P + 8), dict(ld=1020), dict(ld_head=132), dict(out_ld=1028),
                                              dict(out_ld_head=127), dict(out_ld_head=120), dict(out_ld=1016), dict(table=P + 2), dict(lengths=P + 1), dict(starts=P + 2), dict(prefix=P + 3),
                                              dict(rows=-1), dict(rows=2 ** 20 + 1), dict(heads=0), dict(heads=6), dict(heads=1028), dict(seqs=0),
                                              dict(seqs=65536), dict(max_rows=-1), dict(max_rows=13), dict(max_keys=-1), dict(max_keys=577), dict(table_pages=-1),
                                              dict(table_ld=8), dict(prefix_len=-1), dict(prefix_len=321), dict(prefix_pages=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN),
                                              dict(scale=INF), dict(rows=2 ** 20, max_rows=2 ** 20, seqs=65535)], ids=str)
def test_attention_refuses(lib, bad):
    assert attention(lib, **bad) == ec.EC_ERR_ARG
    assert lib.ec_last_error(None)


@pytest.mark.parametrize("bad", [dict(max_keys=2 ** 30 + 1), dict(prefix_len=2 ** 30 + 1), dict(scale=2e38)], ids=str)
def test_attention_refuses_what_does_not_fit(lib, bad):
    assert attention(lib, **dict(page=256, pages=1000, table_pages=2 ** 23, table_ld=2 ** 23, prefix_pages=2 ** 23) | bad) == ec.EC_ERR_ARG
    assert lib.ec_last_error(None)


def test_attention_workspace(lib):
    c = cache()
    for rows, seqs, keys, prefix in ((1, 1, 5000, 0), (3, 3, 100, 5000), (4, 4, 40, 1)):
        cfg = ec.ec_kv_attention_cfg(rows, 8, seqs, 1, keys, 100, 100, prefix, 0, 0.1, 100)
        need = lib.ec_kv_attention_workspace_bytes(C.byref(c), C.byref(cfg))
        assert need > 0
        args = dict(rows=rows, seqs=seqs, max_rows=1, max_keys=keys, table_pages=100, prefix_pages=100, prefix_len=prefix, table_ld=100)
        assert attention(lib, size=need - 1, **args) == attention(lib, ws=None, **args) == attention(lib, ws=P + 64, **args) == ec.EC_ERR_WORKSPACE
    for none in (dict(rows=0, max_rows=0), dict(max_rows=0)):
        assert attention(lib, q=None, out=None, lengths=None, ws=None, size=0, data=None, **none) == ec.EC_OK


def test_the_binding_refuses():
    plan = ec.RotaryPlan(torch.zeros(32, dtype=torch.float64), 64, False, 1.0)
    c = ec.kv_cache(3, 2, 64, 32, device="cpu")
    x, at = torch.zeros((4, 2, 64)), torch.zeros(4, dtype=torch.int32)
    q, table, lengths = torch.zeros((4, 6, 64), dtype=torch.bfloat16), torch.zeros((2, 1), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: ec.rotary(x, at, plan), lambda: ec.kv_write(c, x, x, at), lambda: ec.kv_read(c, at),
                 lambda: ec.kv_attention(q, c, table, lengths)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    starts = torch.zeros(3, dtype=torch.int32)
    for call in (lambda: ec.rotary(x.half(), at, plan), lambda: ec.rotary(x[0], at, plan), lambda: ec.rotary(x, at[:3], plan), lambda: ec.rotary(x, at.long(), plan),
                 lambda: ec.rotary(x.transpose(1, 2), at, plan), lambda: ec.rotary(x, at, plan, out=x.bfloat16()), lambda: ec.rotary(x, at, plan, out=x[:3]),
                 lambda: ec.rotary(x, at, plan._replace(dim=32)), lambda: ec.rotary(x, at, plan._replace(turns=plan.turns.float())),
                 lambda: ec.rotary(x, torch.zeros(8, dtype=torch.int32)[::2], plan),
                 lambda: ec.kv_write(c, x, x[:3], at), lambda: ec.kv_write(c, x, x.bfloat16(), at), lambda: ec.kv_write(c, x[:, :1], x[:, :1], at),
                 lambda: ec.kv_write(c, x[..., ::2], x[..., ::2], at), lambda: ec.kv_write(c, x, x, at.long()), lambda: ec.kv_write(c, x.half(), x.half(), at),
                 lambda: ec.kv_read(c, at, torch.float16), lambda: ec.kv_read(c, at[None]), lambda: ec.kv_read(c, at.long()),
                 lambda: ec.kv_attention(q.float(), c, table, lengths), lambda: ec.kv_attention(q[..., :32], c, table, lengths),
                 lambda: ec.kv_attention(q[:3], c, table, lengths), lambda: ec.kv_attention(q, c, table.long(), lengths),
                 lambda: ec.kv_attention(q, c, table, lengths[:1]), lambda: ec.kv_attention(q, c, table, lengths, starts[:2]),
                 lambda: ec.kv_attention(q, c, table, lengths, max_rows=1), lambda: ec.kv_attention(q, c, table, lengths, max_keys=-1),
                 lambda: ec.kv_attention(q, c, table, lengths, prefix=table), lambda: ec.kv_attention(q, c, table, lengths, prefix_len=-1),
                 lambda: ec.kv_attention(q, c, table, lengths, out=q.float()), lambda: ec.kv_attention(q, c, torch.zeros((2, 8), dtype=torch.int32)[:, ::2], lengths),
                 lambda: ec.kv_cache(3, 2, 96), lambda: ec.kv_cache(3, 2, 64, 16), lambda: ec.kv_cache(0, 2, 64), lambda: ec.kv_cache(3, 2, 64, dtype=torch.float16)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ec.EcError):
        ec.rotary_plan(7, device="cpu")
    assert binding._cache_struct(torch, c).pages == 3
    for data in (c.data[:-1], c.data.float(), c.data[::2]):
        with pytest.raises(ValueError, match="kv_cache"):
            binding._cache_struct(torch, c._replace(data=data))


def test_the_plain_quantiser_of_the_tests():
    """its codes against torch's conversion, which rounds the same way"""
    from tests.kv_reference import E4M3, kept
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn)
    assert np.array_equal(codes.double().numpy(), E4M3)
    x = torch.randn((50, 128), dtype=torch.float64) * torch.exp(4 * torch.randn((50, 1), dtype=torch.float64))
    x = x.float().double()
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / 448))
    want = torch.ldexp(torch.ldexp(x, -e).float().to(torch.float8_e4m3fn).double(), e)
    assert np.array_equal(kept(x.numpy(), "e4m3"), want.numpy())
    assert np.array_equal(kept(x.numpy(), "bf16"), x.bfloat16().double().numpy())
