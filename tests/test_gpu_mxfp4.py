"""Matrices in microscaled 4-bit floating point: to and from it bit for bit, and products against 64 bits, through the binding.

Products of codes, and of codes with bfloat16 values, are exact in float32 and sums are float32: a matrix instruction adds 32 (128 in
4 bits) products to a running sum, each addition off by at most 2^-23 of a partial sum, which the sum of the magnitudes S bounds.  K / 32 + 32
(K / 128 + 128) such additions, and 16 more for joining parts of K, make (K / 32 + 144) 2^-23 S; bfloat16 results are rounded once
(2^-8 of the value)."""
import itertools

import numpy as np
import pytest
import torch

import paper_2603_18489_amd as ec

pytestmark = pytest.mark.gpu

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def quantize(x):
    """codes and scale bytes by the definition, in 64 bits: the nearest of the eight magnitudes, the even code on ties"""
    rows, k = x.shape
    v = x.astype(np.float64).reshape(rows, k // 32, 32)
    good = np.isfinite(v).all(axis=-1)
    v = np.where(good[..., None], v, 0.0)
    top = np.abs(v).max(axis=-1)
    e = np.floor(np.log2(np.where(top > 0, top, 2.0 ** -200)))
    e = np.where(2.0 ** (e + 1) <= top, e + 1, np.where(2.0 ** e > top, e - 1, e))     # (log2 rounds)
    e = np.maximum(e - 2, -127)
    y = np.minimum(np.abs(v) / 2.0 ** e[..., None], 6.0)
    far = np.abs(y[..., None] - E2M1[:8])
    far -= 1e-9 * (np.arange(8) % 2 == 0)          # (nearer by less than any distance between two)
    code = far.argmin(axis=-1) | (np.signbit(v) << 3)
    code = np.where(good[..., None], code, 0).reshape(rows, k)
    return (code[:, ::2] | code[:, 1::2] << 4).astype(np.uint8), np.where(good, e + 127, 255).astype(np.uint8)


def values(codes, scales):
    v = E2M1[np.stack((codes & 15, codes >> 4), axis=-1).reshape(len(codes), -1)]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, axis=1)


def matrix(rows, k, seed=0, spread=0.0):
    rng = np.random.default_rng(seed + 1000 * rows + k)
    return (rng.standard_normal((rows, k)) * np.exp(spread * rng.standard_normal((rows, k)))).astype(np.float32)


def on_gpu(x, dtype="f32", pad=0):
    buf = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=DTYPES[dtype], device="cuda")
    buf[:, :x.shape[1]] = torch.from_numpy(x).cuda()
    return buf[:, :x.shape[1]]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k,pad", [(1, 32, 0), (3, 64, 1), (7, 96, 5), (33, 1056, 0), (5, 4096, 8), (1000, 32, 0), (130, 3584, 32)])
def test_quantize_is_the_definition(rows, k, pad, dtype):
    x = on_gpu(matrix(rows, k, spread=2.0), dtype, pad)
    q = ec.mxfp4_quantize(x)
    codes, scales = quantize(x.float().cpu().numpy())
    assert np.array_equal(q.codes.cpu().numpy(), codes) and np.array_equal(q.scales.cpu().numpy(), scales)
    for out in ("f32", "bf16"):
        back = ec.mxfp4_dequantize(q, DTYPES[out])
        assert back.dtype == DTYPES[out]
        assert np.array_equal(back.double().cpu().numpy(), values(codes, scales))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_ends_ties_and_values_that_are_none(dtype):
    """Halfway values of every binade, the ends of the type, subnormals, zeros of both signs, and blocks with an infinity or a NaN."""
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, 7.5, 4, 3.25, 0.125, 0.0, -0.0, -0.25, -0.75, -5])
    rows = []
    for e in (-149, -140, -133, -130, -128, -127, -126, -125, -124, -100, -1, 0, 1, 60, 124, 125):
        row = np.zeros(32)
        row[:18] = ties * 2.0 ** e
        row[20] = 7.75 * 2.0 ** e           # (keeps the block's scale at 2^e)
        rows.append(row)
    rows += [np.zeros(32), -np.zeros(32), np.full(32, 2.0 ** 127 * 1.98)]
    for bad in (np.inf, -np.inf, np.nan):
        for at in (0, 13, 31):
            row = np.ones(32)
            row[at] = bad
            rows.append(row)
    with np.errstate(over="ignore"):
        x = on_gpu(np.concatenate((np.array(rows), np.ones((len(rows), 32))), axis=1).astype(np.float32), dtype)
    q = ec.mxfp4_quantize(x)
    codes, scales = quantize(x.float().cpu().numpy())
    assert np.array_equal(q.codes.cpu().numpy(), codes) and np.array_equal(q.scales.cpu().numpy(), scales)
    assert (scales[:, 1] == 125).all() and (scales[-9:, 0] == 255).all()      # (the block beside it is its own)
    back = ec.mxfp4_dequantize(q).double().cpu().numpy()
    np.testing.assert_array_equal(back, values(codes, scales))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_code_of_every_scale_comes_back(dtype):
    """256 scales, all pairs of codes; 6 * 2^126 and beyond overflow to an infinity."""
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 16, axis=1)
    got = ec.mxfp4_dequantize(ec.Mxfp4(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()), DTYPES[dtype])
    want = values(codes, scales)
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
    np.testing.assert_array_equal(got.double().cpu().numpy(), want)


def product(x, w):
    """x W^T in 64 bits, and the sum of the magnitudes"""
    x, w = torch.from_numpy(x).cuda(), torch.from_numpy(w).cuda()
    return (x @ w.t()).cpu().numpy(), (x.abs() @ w.abs().t()).cpu().numpy()


def check_linear(m, n, k, act, out, seed=0, pad=0):
    w = quantize(matrix(n, k, seed + 1, 0.5))
    wq = ec.Mxfp4(*(torch.from_numpy(a).cuda() for a in w))
    packed = ec.mxfp4_pack(wq)
    assert (packed.n, packed.k) == (n, k)
    x = on_gpu(matrix(m, k, seed), "bf16", pad)
    arg, xv = x, x.double().cpu().numpy()
    if act == "mxfp4":
        arg = ec.mxfp4_quantize(x)
        xv = values(*quantize(x.float().cpu().numpy()))
    y = ec.mxfp4_linear(arg, packed, DTYPES[out])
    assert y.shape == (m, n) and y.dtype == DTYPES[out]
    want, size = product(xv, values(*w))
    bound = (k / 32 + 144) * 2.0 ** -23 * size + (2.0 ** -8 * np.abs(want) if out == "bf16" else 0) + 1e-30
    far = np.abs(y.double().cpu().numpy() - want)
    assert (far <= bound).all(), (far / bound).max()
    assert torch.equal(y, ec.mxfp4_linear(arg, packed, DTYPES[out]))      # the same bits again
    return y


SIZES = [(1, 16, 32), (1, 1, 64), (3, 7, 96), (5, 17, 128), (16, 100, 160), (17, 33, 4096), (2, 2000, 512), (33, 48, 1056),
         (34, 4096, 4096), (48, 96, 992), (64, 1000, 2048), (65, 130, 640), (96, 257, 1184), (97, 256, 1024), (128, 128, 128),
         (129, 300, 544), (255, 129, 96), (300, 1111, 2080), (561, 640, 3584), (1030, 520, 288)]


@pytest.mark.parametrize("act,out", itertools.product(("bf16", "mxfp4"), ("bf16", "f32")))
@pytest.mark.parametrize("m,n,k", SIZES)
def test_linear_against_64_bits(m, n, k, act, out):
    check_linear(m, n, k, act, out)


@pytest.mark.parametrize("act", ["bf16", "mxfp4"])
@pytest.mark.parametrize("m,n,k,pad", [(1, 24576, 4096, 0), (32, 37888, 3584, 64), (1, 64, 18944, 8), (34, 4096, 12288, 0),
                                       (768, 4096, 12288, 8), (2048, 4096, 1024, 0), (700, 12288, 4096, 0)])
def test_linear_at_the_models_sizes(m, n, k, pad, act):
    check_linear(m, n, k, act, "bf16", pad=pad)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(17, 32900, 96), (33, 40001, 160), (64, 49160, 32), (16, 70001, 128), (48, 70004, 480), (5, 98320, 64),
                                   (32, 100100, 224), (9, 131073, 32), (50, 98321, 160), (64, 140001, 96)])
def test_linear_with_few_rows_and_many_features(m, n, k, out):
    check_linear(m, n, k, "bf16", out)


@pytest.mark.parametrize("act", ["bf16", "mxfp4"])
@pytest.mark.parametrize("m,n,k", [(1, 99001, 4096), (4, 33000, 8192), (5, 33000, 8192)])
def test_few_rows_many_features_and_ranges_of_k(m, n, k, act):
    """K is split over blocks where rows lie in registers, and not where waves share them.  The matrix is codes and scales at random."""
    rng = torch.Generator(device="cuda").manual_seed(n)
    codes = torch.randint(0, 256, (n, k // 2), dtype=torch.uint8, device="cuda", generator=rng)
    scales = torch.randint(120, 131, (n, k // 32), dtype=torch.uint8, device="cuda", generator=rng)
    w = ec.Mxfp4(codes, scales)
    x = torch.randn((m, k), device="cuda", generator=rng).bfloat16()
    arg = ec.mxfp4_quantize(x) if act == "mxfp4" else x
    xv = (ec.mxfp4_dequantize(arg) if act == "mxfp4" else x).double()
    y = ec.mxfp4_linear(arg, ec.mxfp4_pack(w), torch.float32)
    wv = ec.mxfp4_dequantize(w).double()
    off = (y.double() - (wv @ xv.t()).t()).abs()
    assert (off <= (k / 32 + 144) * 2.0 ** -23 * (wv.abs() @ xv.abs().t()).t()).all()


@pytest.mark.parametrize("act", ["bf16", "mxfp4"])
@pytest.mark.parametrize("m", [1, 20, 130])
def test_blocks_that_are_none_and_wide_scales(m, act):
    """A NaN block reaches the products of its row and no others; scales from 2^-60 to 2^60 in one row; a zero matrix."""
    k, n = 320, 50
    codes, scales = quantize(matrix(n, k, 5))
    scales = (scales.astype(int) + np.random.default_rng(1).integers(-60, 60, scales.shape)).astype(np.uint8)
    codes[7] = 0
    scales[7] = 0
    scales[11, 3] = 255
    x = on_gpu(matrix(m, k, 6), "bf16")
    if m > 1:
        x[m - 1, 40] = float("nan")
    arg, xv = x, x.double().cpu().numpy()
    if act == "mxfp4":
        arg = ec.mxfp4_quantize(x)
        xv = values(*quantize(x.float().cpu().numpy()))
    y = ec.mxfp4_linear(arg, ec.mxfp4_pack(ec.Mxfp4(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda())), torch.float32)
    y = y.double().cpu().numpy()
    want, size = product(xv, values(codes, scales))
    assert np.array_equal(np.isnan(y), np.isnan(want)) and np.isnan(want[:, 11]).all()
    ok = ~np.isnan(want)
    assert (np.abs(y - want)[ok] <= ((k / 32 + 144) * 2.0 ** -23 * size)[ok]).all()
    assert (y[: max(m - 1, 1), 7] == 0).all()


@pytest.mark.parametrize("act", ["bf16", "mxfp4"])
@pytest.mark.parametrize("m,n,k,ldy", [(1, 30, 128, 33), (40, 50, 256, 64), (200, 130, 160, 131)])
def test_rows_with_gaps_are_left_alone(m, n, k, ldy, act):
    """y of another row stride: what lies between the rows and behind them is not written."""
    lib = ec.load_library()
    packed = ec.mxfp4_pack(ec.mxfp4_quantize(on_gpu(matrix(n, k))))
    x = on_gpu(matrix(m, k, 3), "bf16")
    q = ec.mxfp4_quantize(x)
    size = lib.ec_mx_linear_workspace_bytes(ec.EC_T_MXFP4 if act == "mxfp4" else ec.EC_T_BF16, m, n, k)
    ws = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
    for kind, dtype in ((ec.EC_T_F32, torch.float32), (ec.EC_T_BF16, torch.bfloat16)):
        y = torch.full((m + 3, ldy), 77.0, dtype=dtype, device="cuda")
        args = (q.codes.data_ptr(), q.scales.data_ptr(), ec.EC_T_MXFP4) if act == "mxfp4" else (x.data_ptr(), None, ec.EC_T_BF16)
        rc = lib.ec_mx_linear(*args, m, k, packed.data.data_ptr(), n, k, y.data_ptr(), kind, ldy, ws.data_ptr(), size,
                              torch.cuda.current_stream().cuda_stream)
        assert rc == ec.EC_OK
        assert (y[m:] == 77).all() and (y[:, n:] == 77).all()
        assert torch.equal(y[:m, :n], ec.mxfp4_linear(q if act == "mxfp4" else x, packed, dtype))


def test_no_rows():
    packed = ec.mxfp4_pack(ec.mxfp4_quantize(on_gpu(matrix(20, 64))))
    x = torch.zeros((0, 64), dtype=torch.bfloat16, device="cuda")
    q = ec.mxfp4_quantize(x)
    assert q.codes.shape == (0, 32) and q.scales.shape == (0, 2)
    assert ec.mxfp4_dequantize(q).shape == (0, 64)
    assert ec.mxfp4_linear(x, packed).shape == ec.mxfp4_linear(q, packed).shape == (0, 20)


@pytest.mark.parametrize("m", [1, 34, 300])
@pytest.mark.parametrize("act", ["bf16", "mxfp4"])
def test_streams_and_graphs(m, act):
    """Another current stream, a stream handed over, calls at once, and a captured call replayed on new rows: the same bits."""
    n, k = 2048, 2048
    packed = ec.mxfp4_pack(ec.mxfp4_quantize(on_gpu(matrix(n, k))))
    xs = [on_gpu(matrix(m, k, s), "bf16").contiguous() for s in (1, 2)]
    run = lambda x, **kw: ec.mxfp4_linear(ec.mxfp4_quantize(x, **kw) if act == "mxfp4" else x, packed, **kw)
    ref = [run(x) for x in xs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [run(xs[0]) for _ in range(4)]
    here = [run(xs[1]) for _ in range(4)]
    handed = run(xs[0], stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(g, ref[0]) for g in got + [handed]) and all(torch.equal(h, ref[1]) for h in here)
    graph, x = torch.cuda.CUDAGraph(), xs[0].clone()
    with torch.cuda.graph(graph):
        y = run(x)
    for i in (1, 0, 1):
        x.copy_(xs[i])
        graph.replay()
        eager = run(xs[1 - i])
        torch.cuda.synchronize()
        assert torch.equal(y, ref[i]) and torch.equal(eager, ref[1 - i])


def test_head_in_four_bits_and_tokens_drawn_from_its_logits():
    """The end of a step: the LM head quantised on the device, its product with the block's rows, tokens drawn from the logits
    beside the vocabulary reduction of the same logits."""
    rows, d, V = 32, 512, 32000
    head, h = matrix(V, d, 8), matrix(rows, d, 9)
    packed = ec.mxfp4_pack(ec.mxfp4_quantize(on_gpu(head)))
    x, u = on_gpu(h, "bf16"), torch.rand(rows, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    logits = ec.mxfp4_linear(x, packed, torch.float32)
    tokens, stats = ec.row_sample(logits, u, temperature=0.7, top_p=0.95)
    entropy = ec.row_entropy(logits)
    want, size = product(x.double().cpu().numpy(), values(*quantize(head)))
    assert (np.abs(logits.double().cpu().numpy() - want) <= (d / 32 + 144) * 2.0 ** -23 * size).all()
    from tests.test_gpu_row_sample import draw
    z = logits.cpu().numpy()
    assert tokens.cpu().tolist() == [draw(z[i], u[i].item(), 0.7, 0, 0.95)[0] for i in range(rows)]
    assert (entropy[:, 0].long() == logits.argmax(dim=1)).all()
    greedy, _ = ec.row_sample(logits, u, temperature=0.0)
    assert (greedy == entropy[:, 0].int()).all()


def test_more_than_two_to_the_32_threads():
    """2^32 groups of eight values and some: a launch of its own for what one does not take."""
    rows, k = 2 ** 18 + 3, 131072
    if torch.cuda.mem_get_info()[0] < 180 << 30:
        pytest.skip("180 GiB are needed")
    x = torch.zeros((rows, k), dtype=torch.bfloat16, device="cuda")
    some = [0, 2 ** 17 - 1, 2 ** 17, 2 ** 18 - 1, 2 ** 18, rows - 1]
    x[some] = torch.randn((len(some), k), device="cuda").bfloat16()
    q = ec.mxfp4_quantize(x)
    ref = ec.mxfp4_quantize(x[some])
    assert torch.equal(q.codes[some], ref.codes) and torch.equal(q.scales[some], ref.scales)
    assert all(not q.scales[i:i + 4096].any() for i in (1, 2 ** 17 + 1, 2 ** 18 - 4097))
    x.fill_(1)
    values = ec.load_library().ec_mx_dequantize(q.codes.data_ptr(), q.scales.data_ptr(), rows, k, x.data_ptr(), ec.EC_T_BF16, k,
                                                torch.cuda.current_stream().cuda_stream)
    assert values == ec.EC_OK
    assert torch.equal(x[some], ec.mxfp4_dequantize(ref, torch.bfloat16))
    assert all(not x[i:i + 4096].any() for i in (1, 2 ** 17 + 1, 2 ** 18 - 4097))
    del x
    packed, few = ec.mxfp4_pack(q), ec.mxfp4_pack(ref)
    y = torch.randn((2, k), device="cuda").bfloat16()
    # Another number of features may split K into other ranges, so that float32 sums meet in another order: each of the two results is
    # within (k / 32 + 144) 2^-23 of the products' magnitudes, as everywhere here, and they of each other within twice that.
    size = y.double().abs() @ ec.mxfp4_dequantize(ref).double().abs().t()
    off = (ec.mxfp4_linear(y, packed, torch.float32)[:, some].double() - ec.mxfp4_linear(y, few, torch.float32).double()).abs()
    assert (off <= 2 * (k / 32 + 144) * 2.0 ** -23 * size).all()
    del q, packed
    torch.cuda.empty_cache()


@pytest.mark.parametrize("m", [3, 40, 130])
def test_scales_at_any_byte_and_a_matrix_that_is_not_packed(m):
    n, k = 200, 256
    packed = ec.mxfp4_pack(ec.mxfp4_quantize(on_gpu(matrix(n, k))))
    q = ec.mxfp4_quantize(on_gpu(matrix(m, k, 3), "bf16"))
    ref = ec.mxfp4_linear(q, packed)
    for off in (1, 2, 3):
        scales = torch.zeros(q.scales.numel() + off, dtype=torch.uint8, device="cuda")[off:].view_as(q.scales)
        scales.copy_(q.scales)
        assert torch.equal(ec.mxfp4_linear(ec.Mxfp4(q.codes, scales), packed), ref)
    with pytest.raises(ValueError):
        ec.mxfp4_linear(q, ec.Mxfp4Matrix(packed.data[:-1], n, k))
