"""Tokens drawn from rows of logits (ec_row_sample) against the definition in 64 bits, through the binding.

Tokens are compared for equality: the definition's running sums in 64 bits and the library's differ by less than 1e-11 of a row's
sum, so that a uniform number falls between the two for about one row in a million.  Statistics are quotients of those sums, rounded
to float32 once (2^-24), and an e of 2^-46 c is itself off by at most 2^-47: 2^-23 relative holds for e above 2^-23."""
import numpy as np
import pytest
import torch

import paper_2603_18489_amd as ec
from paper_2603_18489_amd import binding

pytestmark = pytest.mark.gpu


def draw(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """one row in 64 bits: (token, four statistics)"""
    t, p, m = (float(np.float32(v)) for v in (temperature, top_p, min_p))
    if t == 0:
        t, top_k = 1.0, 1
    z = z.astype(np.float64)
    if np.isnan(z).any() or not np.isfinite(z.max()):
        return -1, [np.nan] * 4
    with np.errstate(over="ignore", under="ignore"):
        e = np.exp((z - z.max()) / t)
    order = np.lexsort((np.arange(len(z)), -z))
    order = order[z[order] > -np.inf]
    if top_k:
        order = order[:top_k]
    if p < 1:
        before = np.concatenate(([0.0], np.cumsum(e[order])[:-1]))
        order = order[before < p * e[order].sum()]
    order = np.sort(order[e[order] >= m])
    sums = np.cumsum(e[order])
    u = min(max(float(u), 0.0), float(np.float32(1 - 2.0 ** -24))) if u == u else 0.0
    token = order[min(np.searchsorted(sums, u * sums[-1], side="right"), len(order) - 1)]
    return token, [e[token] / sums[-1], e[token] / e.sum(), len(order), sums[-1] / e.sum()]


def check(z, u, **filters):
    """z: a CUDA matrix, u: numbers"""
    u = np.asarray(u, dtype=np.float32)
    tokens, stats = ec.row_sample(z, torch.from_numpy(u).cuda(), **filters)
    ref = [draw(row, v, **filters) for row, v in zip(z.float().cpu().numpy(), u)]
    assert tokens.cpu().tolist() == [int(r[0]) for r in ref]
    np.testing.assert_allclose(stats.cpu().numpy().reshape(-1, 4), np.array([r[1] for r in ref]).reshape(-1, 4), rtol=2.0 ** -23)
    return tokens.cpu().numpy(), stats.cpu().numpy()


def logits(rows, V, dtype=torch.float32, pad=0, seed=0):
    """rows from nearly flat to nearly decided"""
    rng = np.random.default_rng(seed + V)
    z = rng.standard_normal((rows, V + pad)) * rng.uniform(0.3, 5.0, (rows, 1))
    z[np.arange(rows), rng.integers(0, V, rows)] += rng.uniform(0, 20, rows)
    return torch.from_numpy(z.astype(np.float32)).cuda().to(dtype)[:, :V], rng.random(rows, dtype=np.float32)


FILTERS = [dict(), dict(temperature=0.7), dict(top_k=1), dict(top_k=7), dict(top_k=50, temperature=0.3), dict(top_p=0.9),
           dict(top_p=0.05), dict(top_p=0.999, temperature=1.7), dict(min_p=0.1), dict(min_p=1.0), dict(top_k=300, top_p=0.95, min_p=0.001),
           dict(temperature=2.0, top_p=0.5, min_p=0.02), dict(top_k=10 ** 9), dict(temperature=0.0), dict(temperature=0.0, top_p=0.3)]


@pytest.mark.parametrize("filters", FILTERS, ids=str)
@pytest.mark.parametrize("rows,V,dtype,pad", [(1, 2, "f32", 0), (5, 33, "bf16", 1), (3, 1000, "f32", 3), (9, 4096, "bf16", 0),
                                              (4, 20011, "f32", 1), (3, 50000, "bf16", 5)])
def test_against_the_definition(rows, V, dtype, pad, filters):
    z, u = logits(rows, V, {"f32": torch.float32, "bf16": torch.bfloat16}[dtype], pad)
    check(z, u, **filters)


@pytest.mark.parametrize("filters", [dict(temperature=0.8), dict(temperature=0.2, top_p=0.95), dict(top_p=0.9), dict(top_k=50),
                                     dict(top_k=1000, top_p=0.9, min_p=0.001), dict(min_p=0.05), dict(top_k=60000)], ids=str)
@pytest.mark.parametrize("rows,V,dtype", [(6, 126464, "f32"), (5, 152064, "bf16"), (3, 163840, "f32"), (2, 163839, "bf16")])
def test_full_vocabularies(rows, V, dtype, filters):
    z, u = logits(rows, V, {"f32": torch.float32, "bf16": torch.bfloat16}[dtype], pad=1)
    z[0] = 0.01 * z[0]      # nearly flat: the borders lie 1 / V apart
    check(z, u, **filters)


@pytest.mark.parametrize("V", [2, 64, 4097, 40000, 163840])
def test_equal_logits_go_by_their_ids(V):
    """A constant row, zeros of both signs: the kept tokens are the lowest ids, and u picks among them evenly."""
    u = np.concatenate((np.linspace(0, 0.999, 13), [1 - 2.0 ** -24])).astype(np.float32)
    z = torch.zeros((len(u), V), device="cuda")
    z[:, ::2] = -0.0
    for k in {1, 2, min(V - 1, 5), V - 1, V}:
        tokens, stats = check(z, u, top_k=k)
        assert (tokens == np.floor(u.astype(np.float64) * k)).all() and (stats[:, 2] == k).all()
    tokens, _ = check(z, u, top_p=0.5)
    assert tokens.max() < (V + 1) // 2
    z = torch.full((len(u), V), -7.25, device="cuda", dtype=torch.bfloat16)
    z[:, V // 2] = 1.0
    check(z, u, top_k=V // 2 + 1)


def test_ties_at_the_cut_across_the_whole_row():
    """Few distinct values, so that the cut falls among thousands of equal ones."""
    rng = np.random.default_rng(3)
    z = torch.from_numpy(rng.integers(-3, 4, (6, 60000)).astype(np.float32) * 0.5).cuda()
    u = rng.random(6, dtype=np.float32)
    for filters in (dict(top_k=8570), dict(top_k=20001), dict(top_p=0.31), dict(top_p=0.8, top_k=30000), dict(min_p=0.3)):
        check(z, u, **filters)
        check(z.bfloat16(), u, **filters)


@pytest.mark.parametrize("V", [50, 4096, 70000])
def test_masked_rows(V):
    """-inf and the type's lowest value in masked places; rows without a distribution; the others beside them untouched."""
    z, u = logits(9, V, seed=5)
    low = torch.finfo(torch.float32).min
    z[0, 1::2] = -float("inf")
    z[1] = -float("inf")                       # nothing left
    z[2] = -float("inf")
    z[2, V - 1] = -1e30                        # one left
    z[3, : V - 5] = low
    z[4] = low                                 # flat after all
    z[5, V // 2] = float("nan")
    z[6, V // 3] = float("inf")
    z[7] = float("nan")
    for filters in (dict(), dict(top_k=V - 3), dict(top_k=3), dict(top_p=0.9), dict(min_p=0.2), dict(top_k=V // 2, top_p=0.7, min_p=0.01)):
        tokens, stats = check(z, u, **filters)
        assert (tokens[[1, 5, 6, 7]] == -1).all() and tokens[2] == V - 1


@pytest.mark.parametrize("V", [300, 40000])
def test_uniforms_at_and_past_the_ends(V):
    z, _ = logits(8, V, seed=9)
    u = [0.0, 1 - 2.0 ** -24, 1.0, 5.0, -1.0, float("nan"), float("inf"), 2.0 ** -149]
    z[:, V - 1] = 3.0
    for filters in (dict(), dict(top_k=4), dict(top_p=0.8)):
        tokens, _ = check(z, u, **filters)
    z[:, 0] = z[:, V - 1] = -float("inf")
    tokens, _ = check(z, u)
    assert (tokens[[0, 4, 5]] == 1).all()


@pytest.mark.parametrize("temperature", [1e-38, 1e-3, 1e30])
def test_temperatures_at_the_ends(temperature):
    z, u = logits(5, 5000, seed=11)
    tokens, stats = check(z, u, temperature=temperature)
    if temperature < 1e-30:
        assert (tokens == z.argmax(dim=1).cpu().numpy()).all() and (stats[:, 0] == 1).all()


def test_greedy_is_the_vocabulary_reduction():
    z, u = logits(40, 126464, seed=13)
    tokens, stats = ec.row_sample(z, torch.from_numpy(u).cuda(), temperature=0.0)
    entropy = ec.row_entropy(z)
    assert (tokens == entropy[:, 0].int()).all() and (stats[:, 0] == 1).all()
    # (float32 sums there: the bound of its own tests)
    assert ((stats[:, 1] / entropy[:, 1] - 1).abs() < 4e-6).all()


def test_frequencies():
    """The draws of evenly spaced uniform numbers hit each kept token as often as its probability says, within one."""
    z, _ = logits(1, 500, seed=17)
    n = 20000
    u = (np.arange(n) + 0.5) / n
    tokens, _ = ec.row_sample(z.expand(n, 500).contiguous(), torch.from_numpy(u.astype(np.float32)).cuda(), 1.0, 40, 0.9)
    e = np.exp(z[0].double().cpu().numpy())
    keep = np.argsort(-e)[:40]
    keep = keep[: 1 + np.searchsorted(np.cumsum(e[keep]), 0.9 * e[keep].sum())]
    p = np.zeros(500)
    p[keep] = e[keep] / e[keep].sum()
    assert np.abs(np.bincount(tokens.cpu().numpy(), minlength=500) - n * p).max() <= 1.01


def test_empty_and_many_rows():
    tokens, stats = ec.row_sample(torch.zeros((0, 100), device="cuda"), torch.zeros(0, device="cuda"))
    assert tokens.shape == (0,) and stats.shape == (0, 4)
    z, u = logits(3000, 40, seed=19)
    check(z, u, top_k=12, top_p=0.9)


@pytest.mark.parametrize("V,filters", [(4096, dict(top_k=20, top_p=0.9)), (126464, dict()), (126464, dict(top_p=0.9)),
                                       (126464, dict(top_k=50, min_p=0.01))], ids=str)
def test_streams_and_graphs(V, filters):
    """Another current stream, a stream that is handed over, two calls at once and a captured call, replayed on new logits,
    give the bits of the plain call."""
    z, u = logits(32, V, seed=23)
    z2, u2 = logits(32, V, seed=29)
    u, u2 = torch.from_numpy(u).cuda(), torch.from_numpy(u2).cuda()
    ref, ref2 = ec.row_sample(z, u, **filters), ec.row_sample(z2, u2, **filters)
    same = lambda a, b: all(torch.equal(x, y) for x, y in zip(a, b))
    assert same(ref, ec.row_sample(z, u, **filters))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [ec.row_sample(z, u, **filters) for _ in range(3)]
    other = ec.row_sample(z2, u2, **filters)
    handed = ec.row_sample(z2, u2, stream=side, **filters)
    torch.cuda.synchronize()
    assert all(same(g, ref) for g in got) and same(other, ref2) and same(handed, ref2)
    graph, x, v = torch.cuda.CUDAGraph(), z.clone(), u.clone()
    with torch.cuda.graph(graph):
        out = ec.row_sample(x, v, **filters)
    for a, b, r in ((z2, u2, ref2), (z, u, ref), (z2, u2, ref2)):
        x.copy_(a)
        v.copy_(b)
        graph.replay()
        eager = ec.row_sample(a, b, **filters)
        torch.cuda.synchronize()
        assert same(out, r) and same(eager, r)


def test_columns_and_rows_beyond_are_left_alone():
    V, rows = 1000, 3
    lib = ec.load_library()
    z, u = logits(rows, V, seed=31)
    z = z.contiguous()
    tokens = torch.full((rows + 2,), 77, dtype=torch.int32, device="cuda")
    stats = torch.full((rows + 2, 4), 77.0, device="cuda")
    ws = torch.zeros(lib.ec_row_sample_workspace_bytes(rows, V), dtype=torch.uint8, device="cuda")
    cfg = binding.ec_sample_cfg(1.0, 5, 0.9, 0.0)
    rc = lib.ec_row_sample(z.data_ptr(), ec.EC_T_F32, rows, V, V, torch.from_numpy(u).cuda().data_ptr(), cfg, tokens.data_ptr(),
                           stats.data_ptr(), ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert rc == ec.EC_OK
    assert (tokens[rows:] == 77).all() and (stats[rows:] == 77).all() and (tokens[:rows] >= 0).all()


@pytest.mark.parametrize("filters", [dict(temperature=0.8), dict(top_k=50, top_p=0.9), dict(min_p=0.05)], ids=str)
def test_more_rows_than_are_drawn_at_a_time(filters):
    """Rows past 1024 in long rows: each the same as by itself among few."""
    V, rows = 17001, 2100
    z = torch.randn((rows, V), device="cuda") * 3
    u = torch.rand(rows, device="cuda")
    tokens, stats = ec.row_sample(z, u, **filters)
    for lo in (0, 1000, 1023, 1024, 2040, 2090):
        few, of_few = ec.row_sample(z[lo:lo + 10], u[lo:lo + 10].contiguous(), **filters)
        assert torch.equal(tokens[lo:lo + 10], few)
        torch.testing.assert_close(stats[lo:lo + 10], of_few, rtol=2.0 ** -22, atol=0)
    check(z[1020:1030], u[1020:1030].cpu().numpy(), **filters)


def test_a_top_k_beyond_32_bits_is_all():
    z, u = logits(4, 5000)
    u = torch.from_numpy(u).cuda()
    for a, b in zip(ec.row_sample(z, u, top_k=2 ** 32 + 5), ec.row_sample(z, u)):
        assert torch.equal(a, b)
    with pytest.raises(ec.EcError):
        ec.row_sample(z, u, top_k=-2 ** 32 + 5)


@pytest.mark.parametrize("V", [4095, 4096, 4097, 4200, 8191, 8192, 8193, 16384, 16385, 20481])
@pytest.mark.parametrize("filters", [dict(), dict(top_k=4, top_p=0.99), dict(top_p=0.7), dict(min_p=2.0 ** -50), dict(top_k=4095), dict(top_k=16383)], ids=str)
def test_around_the_longest_row_of_one_block(V, filters):
    z, u = logits(3, V)
    check(z, u, **filters)


def test_more_kept_of_the_top_k_than_are_listed():
    """Flat rows in which top-k, and top-p among these, end far down."""
    z = torch.randn((3, 60000), device="cuda") * 0.01
    check(z, [0.1, 0.5, 0.999], top_k=40000, top_p=0.9)
    check(z.bfloat16(), [0.1, 0.5, 0.999], top_k=40000, top_p=0.9, min_p=0.97)


@pytest.mark.parametrize("filters", [dict(top_k=1000), dict(top_k=200, top_p=0.9), dict(top_p=0.8), dict(min_p=0.2), dict(min_p=0.2, top_k=300)], ids=str)
@pytest.mark.parametrize("order", ["falling", "rising", "one place", "every part alike"])
def test_where_the_largest_logits_lie(order, filters):
    """All in one part of a row, which lists only some, or as many in each."""
    z, u = logits(3, 90000, seed=3)
    if order == "one place":
        z = z.clone()
        z[:, 20000:20400] += 8
    elif order == "every part alike":
        z = z[:, :4096].repeat(1, 22)[:, :90000]
    else:
        z = z.sort(dim=1, descending=order == "falling").values
    check(z, u, **filters)
    check(z.repeat(30, 1)[:90].bfloat16(), np.resize(u, 90), **filters)
