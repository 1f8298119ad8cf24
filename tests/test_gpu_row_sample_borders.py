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


SHARES = [0.0, 0.125, 0.25, 0.5, 0.625, 0.75, 0.875]


@pytest.mark.parametrize("temperature", [1.0, 0.7, 0.2])
@pytest.mark.parametrize("level", [0.0, 1.0, -7.25, 0.3, 11.1, -1000.7])
@pytest.mark.parametrize("V,kept", [(4096, 4096), (5000, 5000), (12288, 12288), (12288, 4000), (60000, 5600), (100000, 100000), (163840, 65536)])
def test_equal_logits_at_whole_shares(V, kept, level, temperature):
    """All that is finite alike: top_p 0.5 keeps half exactly, and a number u that is a share of the tokens kept takes the one behind them."""
    z = torch.full((len(SHARES), V), -INF, device="cuda")
    at = np.sort(np.random.default_rng(V).permutation(V)[:kept])
    z[:, at] = level
    for n, filters in ((kept, dict()), (kept // 2, dict(top_p=0.5)), (kept // 4, dict(top_p=0.25, min_p=0.5)), (kept, dict(min_p=0.3)), (kept - 1000, dict(top_k=kept - 1000)),
                       (kept // 4, dict(top_k=kept // 2, top_p=0.5))):
        tokens, stats = check(z, SHARES, temperature=temperature, **filters)
        assert (stats[:, 2] == n).all() and (tokens == at[np.floor(np.array(SHARES) * n).astype(int)]).all()


def test_a_token_past_the_top_k_is_not_drawn():
    """Tokens 32 T below the largest weigh 2^-46 each; with u = 0 the lowest id that is kept is taken, and no lower one that top-k leaves out."""
    z = torch.full((3, 5000), -100.0, device="cuda")
    z[:, 0] = -32.2
    z[:, 1:3001] = -32.1
    z[:, 4000] = 0
    tokens, _ = check(z, [0.0, 0.5, 0.999], top_k=2000)
    assert tokens.tolist() == [1, 4000, 4000]
