"""Scores that are far from zero, where one rounding of the scaled maximum is many units of the exponent: every product and sum of the scores here is
exact in float32, so that the definition in 64 bits holds however large they are.  Scores that are infinite."""
import numpy as np
import pytest
import torch

import paper_2603_18489_amd as ec
from tests.kv_reference import HALF
from tests.test_gpu_kv_attention import Batch, ints

pytestmark = pytest.mark.gpu

SHAPES = [  # rows and keys of the sequences, heads, kv heads, head dim, page, prefix
    ([1], [1000], 8, 2, 128, 64, 0), ([2, 1], [5000, 70], 4, 4, 64, 64, 0), ([20, 7], [300, 33], 4, 2, 128, 32, 0), ([130, 40], [200, 1000], 2, 2, 64, 64, 0),
    ([150], [2000], 2, 1, 128, 128, 0), ([1] * 9, [3, 0, 40, 12, 65, 1, 31, 33, 8], 8, 2, 128, 64, 700), ([3, 2], [90, 500], 4, 4, 64, 32, 1300),
    ([70, 90], [100, 30], 2, 2, 128, 32, 333)]


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("scale", [1e-40, 2.0 ** -30, 2.0 ** -10, 2.0 ** -7, 1.0, 2.0 ** 20, 1e30])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_scores_far_from_zero(shape, scale, cache):
    counts, lengths, heads, kv_heads, hd, page, prefix = shape
    b = Batch(counts, lengths, heads, kv_heads, hd, page, cache, prefix, seed=3)
    rng = np.random.default_rng(17)
    # keys: 0 or 2^13 beside 0 to 15; queries: what makes scores of a multiple m of base + 1024 n of them
    total = len(b.every)
    base, n = rng.integers(0, 2, (total, kv_heads)), rng.integers(0, 16, (total, kv_heads))
    k = np.zeros((total, kv_heads, hd), dtype=np.float32)
    k[..., 5], k[..., hd - 2] = base * 2.0 ** 13, n
    v = rng.standard_normal((total, kv_heads, hd)).astype(np.float32)
    ec.kv_write(b.cache, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), b.every)
    held_k, held_v = (t.double().cpu().numpy() for t in ec.kv_read(b.cache, b.every, torch.float32))
    assert np.array_equal(held_k, k)
    rows = sum(counts)
    m = rng.choice([1.0, -1.0, 2.0 ** -30, -2.0 ** -14, 0.0], (rows, heads))
    m[0, 0], m[-1, -1] = 1.0, -1.0
    q = np.zeros((rows, heads, hd), dtype=np.float32)
    q[..., 5], q[..., hd - 2] = m * 2.0 ** 20, m * 2.0 ** 10
    out = b.call(q=torch.from_numpy(q).cuda().bfloat16(), scale=scale).double().cpu().numpy()
    cuts = np.cumsum([0] + list(lengths) + [prefix])
    for i in range(len(counts)):
        at = np.concatenate((np.arange(cuts[-2], cuts[-1]), np.arange(cuts[i], cuts[i + 1]))).astype(int)
        for r in range(b.starts[i], b.starts[i + 1]):
            for h in range(heads):
                g = h // (heads // kv_heads)
                s = m[r, h] * (base[at, g] * 2.0 ** 33 + 1024.0 * n[at, g])
                if len(s) == 0:
                    assert (out[r, h] == 0).all()
                    continue
                p = np.exp(np.maximum((s - s.max()) * np.float64(np.float32(scale)), -1000.0))
                w = p / p.sum()
                want, spread = w @ held_v[at, g], w @ np.abs(held_v[at, g])
                # probabilities to bfloat16; exponents of up to 150 (what is further away is 0 either way) after some 8 roundings to float32, above and
                # below the line; the exponential itself (2^-22); sums over the keys; the result to bfloat16
                e = HALF["bf16"] + 2 * (8 * 150 * HALF["f32"] + 2.0 ** -22 + (len(s) / 8 + 16) * HALF["f32"])
                bound = e * spread + HALF["bf16"] * (np.abs(want) + e * spread) + 1e-38
                far = np.abs(out[r, h] - want)
                assert (far <= bound).all(), (i, r, h, m[r, h], (far / bound).max(), out[r, h][:4], want[:4])


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_infinite_scores(shape, cache):
    """a query with scores of +infinity is NaN, one with -infinity alone zeros, and the others of its tile stay right"""
    counts, lengths, heads, kv_heads, hd, page, prefix = shape
    b = Batch(counts, lengths, heads, kv_heads, hd, page, cache, prefix, seed=5)
    keys = [np.concatenate((b.k[-1], x)) for x in b.k[:-1]]
    clean = b.call()
    b.check(clean)
    for value in (float("inf"), float("-inf")):
        q = b.q.clone()
        of = [(int(b.starts[i]), i) for i in range(len(counts))]       # the first row's last head of each sequence
        for r, _ in of:
            q[r, heads - 1, 3] = value
        out = b.call(q=q)
        for r, i in of:
            s = (value * np.sign(keys[i][:, kv_heads - 1, 3]))
            got = out[r, heads - 1]
            if len(s) and (np.isnan(s).any() or s.max() == np.inf):
                assert torch.isnan(got).all()
            else:
                assert (got == 0).all()
            out[r, heads - 1] = clean[r, heads - 1]
        b.check(out)
    # all keys on one side
    k, v = (t.clone() for t in ec.kv_read(b.cache, b.every, torch.float32))
    k[..., 3] = -k[..., 3].abs() - 0.25
    ec.kv_write(b.cache, k, v, b.every)
    q = torch.zeros_like(b.q)
    q[..., 3] = float("inf")
    assert (b.call(q=q) == 0).all()
    q[..., 3] = float("-inf")
    assert torch.isnan(b.call(q=q)[[int(b.starts[i]) for i in range(len(counts)) if prefix + lengths[i]]]).all()
