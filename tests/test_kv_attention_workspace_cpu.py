"""Workspace of the attention over a paged cache: one for so many rows, sequences, keys and prefix keys serves fewer of each."""
import ctypes as C
import itertools
import random

import pytest

import paper_2603_18489_amd as ec


def need(lib, heads, kv_heads, hd, rows, seqs, max_rows, keys, prefix):
    c = ec.ec_kv_cache(None, ec.EC_T_E4M3, 10, 64, kv_heads, hd)
    cfg = ec.ec_kv_attention_cfg(rows, heads, seqs, max_rows, keys, 2 ** 24, 2 ** 24, prefix, 0, 0.1, 2 ** 24)
    return lib.ec_kv_attention_workspace_bytes(C.byref(c), C.byref(cfg))


def fits(heads, kv_heads, hd, rows, seqs, max_rows):
    return rows <= 2 ** 20 and (max_rows * (heads // kv_heads) + 15) // 16 * seqs * kv_heads <= (2 ** 31 - 1) // 1024


HEADS = [(28, 4, 128), (32, 32, 128), (8, 1, 64), (64, 8, 128), (4, 4, 64)]


@pytest.mark.parametrize("prefix", [0, 1, 5000])
@pytest.mark.parametrize("seqs", [1, 3, 16, 300])
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_it_grows_with_the_rows(heads, seqs, prefix):
    lib = ec.load_library()
    for keys in (100, 1024, 1025, 131072):
        sizes = [need(lib, *heads, seqs * n, seqs, n, keys, prefix) for n in itertools.chain(range(0, 300), range(300, 2200, 37))
                 if fits(*heads, seqs * n, seqs, n)]
        assert sizes[0] == 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))
        # (ragged: rows at most max_rows each)
        sizes = [need(lib, *heads, rows, seqs, min(rows, 60), keys, prefix) for rows in range(0, 60 * seqs + 1, max(1, seqs // 2))]
        assert all(a <= b for a, b in zip(sizes, sizes[1:]))


@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_it_grows_with_sequences_and_keys(heads):
    lib = ec.load_library()
    rng = random.Random(4)

    def log(most):
        return max(1, min(most, round(2 ** rng.uniform(0, most.bit_length()))))
    for _ in range(4000):
        seqs, n, keys, prefix = log(400), log(1500), log(140000), rng.choice([0, log(40000)])
        rows = rng.choice([seqs * n, rng.randint(n, seqs * n)])
        if not fits(*heads, rows, seqs, n):      # (asks for 0, and is refused)
            continue
        all_ = need(lib, *heads, rows, seqs, n, keys, prefix)
        fewer = min(seqs, log(seqs))
        m = min(n, log(n))
        some = rng.choice([fewer * m, rng.randint(m, fewer * m)])
        if some > rows:
            continue
        assert need(lib, *heads, some, fewer, m, min(keys, log(keys)), min(prefix, rng.choice([0, log(prefix)]) if prefix else 0)) <= all_
        assert need(lib, *heads, rows, seqs, n, min(keys, log(keys)), prefix) <= all_


def test_where_no_size_has_slices_none_is_needed():
    lib = ec.load_library()
    assert need(lib, 28, 4, 128, 1, 1, 1, 1024, 0) == 0         # few queries, keys of one block
    assert need(lib, 32, 32, 128, 24576, 16, 1536, 480, 0) == 0   # keys of fewer than two slices
