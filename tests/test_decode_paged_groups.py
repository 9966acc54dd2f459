"""The decoding step over a paged cache at the numbers of query heads where its matrix products change: groups of 3 to 16 heads, of 17 to 32, and
larger ones in several parts.  Tolerances: those of tests/test_decode_paged.py."""
import numpy as np
import pytest
import torch

from paged_cases import Cache, ints, normal
from test_decode_paged import check


@pytest.mark.gpu
@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [3, 15, 16, 17, 31, 32, 33, 48])
def test_heads_of_a_group(G, d, mx):
    check(G, 2, 16, d, [47, 0, 300, 1], L=5, La=6, mx=mx, seed=G)
    check(G, 1, 64, d, [6000, 129], L=40, mx=mx, seed=G)


@pytest.mark.gpu
@pytest.mark.parametrize("G", [9, 16, 20, 32])
@pytest.mark.parametrize("d", [64, 128])
def test_rising_logits(G, d):
    """Each head meets its heaviest key in a later block than the one before, so that references rise at different times in different columns."""
    def rows(c, K, V):
        for b, n in enumerate(c.lens):
            for t in range(0, n, 11):
                K[c.table[b, t // 16], 0, t % 16, t // 11 % d] = 4.0 + t / 64

    check(G, 1, 16, d, [500, 77], L=3, change=rows, scale=0.5)
    check(G, 1, 16, d, [500, 77], L=3, mx=True, change=rows, scale=0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_infinite_logits_in_wide_groups(d):
    def some(c, K, V):
        K[:, :, ::3, 0] = float("-inf")

    def all_rows(c, K, V):
        K[:, :, :, 0] = float("-inf")

    ones = lambda Q: Q[:, :, 0].fill_(1.0)
    for G in (10, 20, 40):
        check(G, 1, 16, d, [100, 16, 3000], change=some, change_q=ones)
        O, LSE = check(G, 1, 16, d, [40, 17, 2500], change=all_rows, change_q=ones)
        assert not O.any() and torch.isneginf(LSE).all()


@pytest.mark.gpu
@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("G", [10, 20, 40])
@pytest.mark.parametrize("n", [60, 4000])
def test_nan_in_one_row(G, n, mx):
    """NaN in a key makes its sequence's outputs NaN, NaN in a value one channel of them, and neither touches the other sequences."""
    from paper_2603_15619_amd import moda_attn_decode_paged

    c = Cache(1, 16, 128, [n] * 4, mx=mx)
    Q = normal(torch.Generator().manual_seed(0), 4, G, 128).cuda()
    O, LSE = moda_attn_decode_paged(Q, **c.args(), lengths=ints([n] * 4))
    for pool, at in zip(c.pools, ((c.table[1, 2], 0, 3, 7), (c.table[2, 0], 0, 1, 9))):
        if mx:
            pool.view(torch.uint8)[at] = 0x7f
        else:
            pool[at] = float("nan")
    O2, LSE2 = moda_attn_decode_paged(Q, **c.args(), lengths=ints([n] * 4))
    assert torch.equal(O[[0, 3]], O2[[0, 3]]) and torch.equal(LSE[[0, 2, 3]], LSE2[[0, 2, 3]])
    assert O2[1].isnan().all() and LSE2[1].isnan().all()
    rest = np.delete(np.arange(128), 9)
    assert O2[2, :, 9].isnan().all() and torch.equal(O2[2][:, rest], O[2][:, rest])


@pytest.mark.gpu
@pytest.mark.parametrize("G", [4, 16, 24])
def test_equal_heads_of_a_group(G):
    """A head's result does not depend on its place: a group whose heads are all the same gives every head the same bits."""
    from paper_2603_15619_amd import moda_attn_decode_paged

    c = Cache(2, 32, 64, [900, 31, 0])
    Q = normal(torch.Generator().manual_seed(1), 3, 2, 1, 64).expand(3, 2, G, 64).reshape(3, 2 * G, 64).cuda()
    O, LSE = moda_attn_decode_paged(Q, **c.args(), lengths=ints([900, 31, 0]))
    O, LSE = O.view(3, 2, G, 64), LSE.view(3, 2, G)
    assert torch.equal(O, O[:, :, :1].expand_as(O)) and torch.equal(LSE, LSE[:, :, :1].expand_as(LSE))


@pytest.mark.gpu
@pytest.mark.parametrize("G,Hk,B,d,mx", [(1, 8, 33, 64, False), (1, 2, 128, 128, True), (8, 16, 27, 64, True), (40, 4, 32, 64, False), (2, 1, 700, 64, False)])
def test_lists_of_many_sequences(G, Hk, B, d, mx):
    """Lists that many sequences have, longer than what short calls take, with sequences of nothing and of less than their list among them."""
    rng = np.random.default_rng(B)
    n, R = 180, 16
    lens = [int(x) for x in rng.integers(0, 40 * R, B)]
    lens[0], lens[1], lens[B - 1] = 200 * R, 0, 200 * R - 5
    sel = np.full((B, Hk, n), -1, dtype=np.int32)
    for b in range(B):
        pages = -(-lens[b] // R)
        for g in range(Hk):
            some = np.sort(rng.permutation(pages)[:n])
            sel[b, g, :len(some)] = some
    sel[2, 0] = -1
    check(G, Hk, R, d, lens, L=3, mx=mx, selected=sel, seed=B)
