"""Pins of the fp64 definitions on a paged cache: the definitions on contiguous caches, the library's softmax, a literal bound over every row."""
import numpy as np
import pytest
import torch

from oracle import cache_ref as C
from oracle import moda_ref as M
from oracle import paged_ref as P


def cache(seed, lens, Hk, R, d, spare=3):
    """(K, V [B, Hk, longest, d], their pools and table in a shuffled order)"""
    rng = np.random.default_rng(seed)
    T = max(lens)
    K, V = (rng.standard_normal((len(lens), Hk, T, d)) for _ in range(2))
    pages = [-(-n // R) for n in lens]
    order = rng.permutation(sum(pages) + spare)
    table = np.full((len(lens), max(pages) + 2), -1)
    for b, n in enumerate(pages):
        table[b, :n] = order[sum(pages[:b]):sum(pages[:b]) + n]
    pools = [np.full((len(order), Hk, R, d), np.nan) for _ in range(2)]
    written = P.append(K, V, *pools, table, lens)
    assert len(written) == len(set(written)) == sum(lens)
    return rng, K, V, pools, table


@pytest.mark.parametrize("L", [0, 3])
def test_decoding_over_pages_is_decoding_over_their_rows(L):
    lens = [40, 1, 16, 33]
    rng, K, V, pools, table = cache(0, lens, 2, 16, 64)
    Q = rng.standard_normal((4, 6, 64))
    depth = [rng.standard_normal((4, 2, L, 64)) if L else None for _ in range(2)]
    got, want = P.decode(Q, *pools, table, *depth, lengths=lens), C.decode_step(Q, None, None, K, V, *depth, lengths=lens)
    for name in ("O", "LSE", "mag", "logit"):
        assert np.allclose(got[name], want[name], rtol=1e-13, atol=1e-13), name


def test_decoding_over_all_rows_is_the_last_row_of_the_forward():
    rng, K, V, pools, table = cache(1, [37], 2, 16, 64)
    Q, depth = rng.standard_normal((1, 4, 37, 64)), [rng.standard_normal((1, 2, 37, 3, 64)) for _ in range(2)]
    O, LSE = M.fwd(Q, K, V, *depth)
    r = P.decode(Q[:, :, -1], *pools, table, *(x[:, :, -1] for x in depth), lengths=[37])
    assert np.allclose(r["O"], O[:, :, -1], atol=1e-12) and np.allclose(r["LSE"], LSE[:, :, -1], atol=1e-12)


def test_chosen_and_missing_pages_are_a_mask_on_the_rows():
    """The library's softmax over all rows, with those of pages that the list leaves out, or that are gone, at -inf."""
    lens, R = [70, 16], 16
    rng, K, V, pools, table = cache(2, lens, 2, R, 64)
    Q = rng.standard_normal((2, 2, 64))
    table[0, 3] = -1
    selected = np.array([[[4, 0, -1], [3, 2, 1]], [[0, 7, -1], [-1, -1, 5]]])
    r = P.decode(Q, *pools, table, lengths=lens, selected=selected)
    for b in range(2):
        for g in range(2):
            keep = np.array([t // R in selected[b, g] and table[b, t // R] >= 0 for t in range(lens[b])])
            if not keep.any():
                assert not r["O"][b, g].any() and r["LSE"][b, g] == -np.inf
                continue
            s = torch.tensor(K[b, g, :lens[b]] @ Q[b, g] / 8.0).masked_fill(torch.tensor(~keep), float("-inf"))
            assert np.allclose((torch.softmax(s, 0)[:, None] * torch.tensor(V[b, g, :lens[b]])).sum(0).numpy(), r["O"][b, g], atol=1e-13)
            assert abs(torch.logsumexp(s, 0).item() - r["LSE"][b, g]) < 1e-13
    assert r["LSE"][1, 1] == -np.inf


@pytest.mark.parametrize("mx", [False, True])
def test_rows_come_back(mx):
    lens, R = [50, 0, 17], 16
    rng = np.random.default_rng(3)
    K, V = (rng.standard_normal((3, 2, 50, 64)) for _ in range(2))
    pools, table = [np.full((9, 2, R, 64), np.nan) for _ in range(2)], np.array([[8, 1, 6, 2], [-1] * 4, [0, 5, 7, 99]])
    bounds = np.zeros((9, 2, 2, 64))
    P.append(K, V, *pools, table, lens, mx=mx, bounds=bounds)
    out = [np.full((3, 2, 50, 64), 7.0) for _ in range(2)]
    P.read(*pools, table, *out, lens)
    for x, y in zip((K, V), out):
        x = P.quantise(x)[0] if mx else x
        for b, n in enumerate(lens):
            assert np.array_equal(y[b, :, :n], x[b, :, :n]) and np.all(y[b, :, n:] == 7.0)
    x = P.quantise(K)[0] if mx else K
    assert np.array_equal(bounds[6, :, 0], x[0, :, 32:48].min(1)) and np.array_equal(bounds[2, :, 1], x[0, :, 48:50].max(1))
    # row by row as in a prompt at once
    again, bounds2 = [np.full((9, 2, R, 64), np.nan) for _ in range(2)], np.full((9, 2, 2, 64), 5.0)
    for t in range(50):
        P.append(K[:, :, t:t + 1], V[:, :, t:t + 1], *again, table, [min(n, t + 1) for n in lens], [int(t < n) for n in lens], mx=mx, bounds=bounds2)
    assert all(np.array_equal(a, b, equal_nan=True) for a, b in zip(pools, again))
    used = [8, 1, 6, 2, 0, 5]
    assert np.array_equal(bounds[used], bounds2[used])


def test_a_score_bounds_the_sum_of_a_groups_logits():
    lens, R = [64], 16
    rng, K, V, pools, table = cache(4, lens, 1, R, 64)
    Q = rng.standard_normal((1, 3, 64))
    bounds = np.stack([pools[0].min(2), pools[0].max(2)], 2)
    scores = []
    for p in range(4):
        lo, hi = bounds[table[0, p], 0]
        s = sum(np.maximum(q * lo, q * hi).sum() for q in Q[0])  # head by head, channel by channel the larger product
        assert (K[0, 0, p * R:p * R + R] @ Q[0].sum(0)).max() <= s
        scores.append(s)
    got = P.select(Q, bounds, table, 2, R, lens, first=0, recent=0)
    assert got.tolist() == [[sorted(np.argsort(scores)[-2:].tolist())]]
    got = P.select(Q, bounds, table, 2, R, lens, first=1, recent=1)
    assert got.tolist() == [[[0, 3]]]
