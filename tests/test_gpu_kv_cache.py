"""A paged cache of keys and values: what is written and read back, value for value against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2603_18489_amd as ec
from tests.kv_reference import E4M3, kept

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def values(rng, rows, heads, hd, dtype):
    x = rng.standard_normal((rows, heads, hd)) * np.exp(3 * rng.standard_normal((rows, heads, 1)))
    x[rng.random(x.shape) < 0.02] = 0
    return torch.from_numpy(x.astype(np.float32)).cuda().to(DTYPES[dtype])


def equal(got, want):
    assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,heads,hd,page,how", [(1, 1, 64, 32, "run"), (1, 4, 128, 64, "run"), (34, 32, 128, 64, "some"), (100, 3, 64, 32, "any"), (100, 3, 128, 256, "shifted"),
                                                    (7, 5, 128, 128, "any"), (1000, 4, 128, 64, "shifted"), (333, 2, 64, 64, "pages"), (2050, 1, 128, 32, "pages"),
                                                    (4000, 7, 64, 128, "some")])
def test_written_and_read(rows, heads, hd, page, how, dtype, cache):
    rng = np.random.default_rng(rows + hd)
    pages = -(-2 * rows // page) + 2
    c = ec.kv_cache(pages, heads, hd, page, DTYPES[cache])
    at = np.arange(rows)
    if how == "shifted":
        at += 13
    if how == "some":
        at = np.sort(rng.permutation(2 * rows)[:rows])
    slots = at
    if how == "any":
        slots = rng.permutation(pages * page)[:rows]
    if how == "pages":
        slots = rng.permutation(pages)[at // page] * page + at % page
    k, v = (values(rng, rows, heads, hd, dtype) for _ in range(2))
    ec.kv_write(c, k, v, ints(slots))
    want = [kept(t.double().cpu().numpy(), cache) for t in (k, v)]
    for out in ("f32", "bf16"):
        for got, ref in zip(ec.kv_read(c, ints(slots), DTYPES[out]), want):
            equal(got, ref)
    # every other slot is as it was
    rest = np.setdiff1d(np.arange(pages * page), slots)
    for got in ec.kv_read(c, ints(rest), torch.float32):
        assert (got == 0).all()
    # in another order, with some that are not there
    order = rng.permutation(rows)
    mixed = slots[order].astype(np.int64)
    gone = rng.random(rows) < 0.3
    mixed[gone] = rng.choice([-1, pages * page, 2 ** 31 - 1, -2 ** 31], gone.sum())
    for got, ref in zip(ec.kv_read(c, ints(mixed), torch.float32), want):
        equal(got, np.where(gone[:, None, None], 0.0, ref[order]))


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
def test_every_code_border_and_extreme(cache):
    """values on, and next to, every border between codes, under powers of two from the least to the largest; infinities, NaN, zeros"""
    middle = (E4M3[1:] + E4M3[:-1]) / 2
    points = np.concatenate((E4M3, middle, np.nextafter(middle.astype(np.float32), 0), np.nextafter(middle.astype(np.float32), 1e9), [0.0, 440, 447.9]))
    rows = []
    for e in (-149, -140, -130, -126, -125, -20, 0, 1, 60, 119):
        for top in (448.0, 447.0, 449.0, 256.0, 257.0, 1e-3):
            x = np.resize(np.float64(points), 4 * 128).reshape(4, 128) * np.tile([1, -1], 64)
            x = np.clip(x, -top, top)
            x[:, 0] = top
            with np.errstate(over="ignore"):
                rows.append((x * 2.0 ** e).astype(np.float32))
    x = np.concatenate(rows)
    special = np.ones((8, 128), dtype=np.float32)
    special[0, 5], special[1, 127], special[2, 0] = np.inf, -np.inf, np.nan
    special[3] = 0
    special[4], special[4, 3] = 1e-45, -1e-45
    special[5, 9] = np.finfo(np.float32).max          # rounds to an infinity in bfloat16
    special[6, :] = -0.0
    x = np.concatenate((x, special))
    n = len(x)
    c = ec.kv_cache(-(-n // 32), 1, 128, 32, DTYPES[cache])
    t = torch.from_numpy(x[:, None, :]).cuda()
    flipped = t.flip(0).contiguous()
    slots = ints(np.arange(n))
    ec.kv_write(c, t, flipped, slots)
    k, v = ec.kv_read(c, slots, torch.float32)
    equal(k, kept(x.astype(np.float64)[:, None, :], cache))
    equal(v, kept(x[::-1].astype(np.float64)[:, None, :], cache))
    assert torch.equal(torch.signbit(k[n - 2]), torch.ones_like(k[n - 2], dtype=torch.bool))


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("rows", [2, 40, 700, 5000])
def test_the_last_of_rows_with_the_same_slot_is_stored(rows, cache):
    rng = np.random.default_rng(rows)
    c = ec.kv_cache(40, 2, 64, 32, DTYPES[cache])
    slots = rng.integers(0, min(1280, max(1, rows // 2)), rows)
    if rows == 5000:
        slots[-64:] = np.arange(64)          # runs that rows far before name too
        slots[:64] = np.arange(64)
    slots[rng.random(rows) < 0.05] = -1
    k, v = (values(rng, rows, 2, 64, "bf16") for _ in range(2))
    ec.kv_write(c, k, v, ints(slots))
    last = {int(s): r for r, s in enumerate(slots) if s >= 0}
    at = np.array(sorted(last))
    picked = torch.tensor([last[int(s)] for s in at], device="cuda")
    for got, src in zip(ec.kv_read(c, ints(at), torch.float32), (k, v)):
        equal(got, kept(src[picked].double().cpu().numpy(), cache))


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
def test_strides_and_what_lies_between(cache):
    rng = np.random.default_rng(3)
    rows, heads, hd = 75, 3, 128
    slots = ints(np.arange(rows))
    a, b = (ec.kv_cache(4, heads, hd, 32, DTYPES[cache]) for _ in range(2))
    wide = torch.randn((rows, 5 * heads, hd + 3), device="cuda").bfloat16()      # rows of queries, keys and values, at odd strides
    k, v = wide[:, heads:2 * heads, 1:1 + hd], wide[:, 2 * heads:3 * heads, 2:2 + hd]
    ec.kv_write(a, k, v, slots)
    ec.kv_write(b, k.contiguous(), v.contiguous(), slots)
    assert torch.equal(a.data, b.data)
    across = torch.randn((heads, rows, hd), device="cuda").transpose(0, 1)
    one = across[:1].expand(rows, heads, hd)
    ec.kv_write(a, across, one, slots)
    ec.kv_write(b, across.contiguous(), one.contiguous(), slots)
    assert torch.equal(a.data, b.data)
    # reading to strides
    lib = ec.load_library()
    import ctypes as C
    st = ec.ec_kv_cache(a.data.data_ptr(), a.kind, a.pages, a.page, heads, hd)
    for dtype, kind in ((torch.float32, ec.EC_T_F32), (torch.bfloat16, ec.EC_T_BF16)):
        for pad in (0, 1, 8):
            k, v = (torch.full((rows + 1, heads + 1, hd + pad), 7.0, dtype=dtype, device="cuda") for _ in range(2))
            ld = (k.stride(0), k.stride(1))
            assert lib.ec_kv_read(C.byref(st), slots.data_ptr(), rows, k.data_ptr(), v.data_ptr(), kind, *ld, *ld,
                                  torch.cuda.current_stream().cuda_stream) == ec.EC_OK
            for got, want in zip((k, v), ec.kv_read(a, slots, dtype)):
                assert torch.equal(got[:rows, :heads, :hd], want)
                got[:rows, :heads, :hd] = 7
                assert (got == 7).all()


def test_a_cache_of_more_than_4_gib():
    c = ec.kv_cache(150000, 4, 128, 32, torch.float8_e4m3fn)
    assert c.data.numel() > 2 ** 32
    slots = np.array([0, 31, 2 ** 22 + 5, 4194303, 4800000 - 1, 4800000 - 32, 4200000])
    rng = np.random.default_rng(0)
    k, v = (values(rng, len(slots), 4, 128, "f32") for _ in range(2))
    ec.kv_write(c, k, v, ints(slots))
    for got, src in zip(ec.kv_read(c, ints(slots), torch.float32), (k, v)):
        equal(got, kept(src.double().cpu().numpy(), "e4m3"))


def test_no_rows_streams_and_a_graph():
    c = ec.kv_cache(4, 2, 64, 32)
    none = torch.empty((0, 2, 64), device="cuda")
    ec.kv_write(c, none, none, ints([]))
    assert ec.kv_read(c, ints([]))[0].shape == (0, 2, 64)
    k, v = torch.randn((10, 2, 64), device="cuda"), torch.randn((10, 2, 64), device="cuda")
    slots, s = ints(np.arange(5, 15)), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ec.kv_write(c, k, v, slots, stream=s)
    got = ec.kv_read(c, slots, torch.float32, stream=s)
    equal(got[0], kept(k.double().cpu().numpy(), "e4m3"))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ec.kv_write(c, k, v, slots)
        out = ec.kv_read(c, slots, torch.float32)
    for i in range(3):
        k.normal_()
        v.normal_()
        slots.copy_(ints(np.arange(5, 15) * 8 % 128 + i))
        graph.replay()
        torch.cuda.synchronize()
        equal(out[0], kept(k.double().cpu().numpy(), "e4m3"))
        equal(out[1], kept(v.double().cpu().numpy(), "e4m3"))
