"""Rows of ec_row_sample whose cut, or whose token, lies at a border: against the definition in 64 bits, as tests/test_gpu_row_sample.py
compares them (tokens and counts for equality, shares to 2^-23)."""
import numpy as np
import pytest
import torch

from tests.test_gpu_row_sample import check

pytestmark = pytest.mark.gpu
INF = float("inf")


def row(V, *levels):
    """(where from, where to, around, spread) a level; -inf elsewhere"""
    rng = np.random.default_rng(V)
    z = np.full(V, -np.inf)
    for lo, hi, mean, spread in levels:
        z[lo:hi] = mean + spread * rng.standard_normal(hi - lo)
    return torch.from_numpy(z.astype(np.float32)).cuda().repeat(3, 1)


FAR = {
    "listed": (5000, (0, 100, 0, 1), (1000, 4900, -50, 0.3)),
    "ranked by one wave": (5000, (30, 31, 0, 0), (40, 100, -45, 1)),
    "ties": (5000, (7, 8, 0, 0), (100, 1100, -40, 0), (2000, 4000, -100, 0)),
    "cut": (60000, (5000, 55000, 0, 0.5), (1000, 4000, -50, 0.3)),
    "too many to list": (60000, (5000, 15000, 0, 0.5), (20000, 30000, -50, 0.3)),
}


@pytest.mark.parametrize("min_p", [1e-14, 1e-16, 1e-20, 2.0 ** -72, 1e-30])
@pytest.mark.parametrize("name", FAR)
def test_top_k_that_ends_past_all_weight_beside_a_small_min_p(name, min_p):
    """Tokens 32 T and more below the largest weigh nothing, but top-k and min-p say how many of them are kept."""
    z = row(*FAR[name])
    heavy, finite = int((z[0] > -30).sum()), int((z[0] > -INF).sum())
    for k in (heavy + 1, (heavy + finite) // 2, finite - 1):
        for temperature in (1.0, 0.5):
            check(z, [0.1, 0.5, 0.999], top_k=k, min_p=min_p, temperature=temperature)
    check(z, [0.1, 0.5, 0.999], top_k=(heavy + finite) // 2, min_p=min_p, top_p=0.9)
