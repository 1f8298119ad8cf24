"""How many bits a probability has: two bfloat16 parts, 2^-16 together, for a sequence's own keys where max_rows times a group's heads is at most 16, and for a
prefix' where all rows times a group's heads are; one, 2^-8, elsewhere.  Scores of small whole numbers are exact in float32, and values that cancel make the
result small beside what is added up, so that the probabilities' bits show."""
import numpy as np
import pytest
import torch

import paper_2603_18489_amd as ec
from tests.kv_reference import HALF
from tests.test_gpu_kv_attention import Batch

pytestmark = pytest.mark.gpu
TWO = 2.0 ** -16

SHAPES = [  # rows and keys of the sequences, heads, kv heads, head dim, page, prefix
    ([1], [1000], 28, 4, 128, 64, 0), ([4], [900], 4, 2, 64, 32, 0), ([1], [5000], 8, 1, 128, 64, 0), ([2, 2, 1], [300, 40, 2000], 4, 1, 128, 64, 0),
    ([16, 3], [64, 77], 2, 2, 64, 32, 0), ([2, 1], [50, 700], 4, 1, 128, 64, 333), ([1, 1], [20, 9], 28, 4, 128, 32, 3000), ([5, 5, 5], [90, 33, 40], 2, 2, 64, 64, 70),
    # (more than 16 queries of the prefix, by one and by many)
    ([1, 1, 1], [50, 400, 30], 24, 4, 128, 64, 500), ([1] * 17, [60] * 17, 4, 4, 64, 32, 200), ([1] * 64, [40] * 64, 14, 2, 128, 64, 1000)]


def to_bf16(x):
    return torch.from_numpy(x.astype(np.float32)).bfloat16().double().numpy()


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_probabilities_of_two_parts(shape, cache):
    counts, lengths, heads, kv_heads, hd, page, prefix = shape
    b = Batch(counts, lengths, heads, kv_heads, hd, page, cache, prefix, seed=11)
    group = heads // kv_heads
    assert max(counts) * group <= 16
    part_of_prefix = TWO if sum(counts) * group <= 16 else HALF["bf16"]
    scale, rng, cuts = 0.0113, np.random.default_rng(1), np.cumsum([0] + list(lengths) + [prefix])
    k = rng.integers(-15, 16, (len(b.every), kv_heads, hd)).astype(np.float64)
    v = rng.standard_normal(k.shape)
    q = rng.integers(-3, 4, (sum(counts), heads, hd)).astype(np.float64)

    def weights(i, r, h):
        at = np.concatenate((np.arange(cuts[-2], cuts[-1]), np.arange(cuts[i], cuts[i + 1]))).astype(int)
        s = np.float64(np.float32(scale)) * (k[at, h // group] @ q[r, h])
        p = np.exp(s - s.max())
        return at, p, s
    # the values of the last sequence' three weightiest own keys cancel what the others add up to for its first row's first head of each group
    last = len(counts) - 1
    for g in range(kv_heads):
        at, p, _ = weights(last, b.starts[last], g * group)
        w = p / p.sum()
        for j in prefix + np.argsort(-w[prefix:])[:3]:
            v[at[j], g] = -(w @ v[at, g] - w[j] * v[at[j], g]) / w[j]
            ec.kv_write(b.cache, *(torch.from_numpy(x.astype(np.float32)).cuda() for x in (k, v)), b.every)
            v = ec.kv_read(b.cache, b.every, torch.float32)[1].double().cpu().numpy()
    assert np.array_equal(ec.kv_read(b.cache, b.every, torch.float32)[0].double().cpu().numpy(), k)
    out = b.call(q=torch.from_numpy(q).cuda().bfloat16(), scale=scale).double().cpu().numpy()
    seen = []
    for i in range(len(counts)):
        for r in range(b.starts[i], b.starts[i + 1]):
            for h in range(heads):
                g = h // group
                at, p, s = weights(i, r, h)
                w = p / p.sum()
                want, spread = w @ v[at, g], w @ np.abs(v[at, g])
                # (exponents after 4 roundings to float32, above and below the line; exponentials and sums, as the reference counts them)
                e = 2 * (4 * HALF["f32"] * 2 * np.abs(s).max() + 2.0 ** -22 + (len(s) / 8 + 16) * HALF["f32"])
                part = np.where(np.arange(len(s)) < prefix, part_of_prefix, TWO)
                off = (part * w) @ np.abs(v[at, g]) + e * spread
                bound = off + HALF["bf16"] * (np.abs(want) + off) + 1e-38
                assert (np.abs(out[r, h] - want) <= bound).all(), (i, r, h, (np.abs(out[r, h] - want) / bound).max())
                if i == last and r == b.starts[last] and h % group == 0:
                    seen.append((np.abs(to_bf16(p) @ v[at, g] / p.sum() - want) / bound).max())
    # with one part some result would be further off
    assert part_of_prefix != TWO or max(seen) > 1, seen
