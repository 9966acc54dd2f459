"""The choice of pages by their key bounds, against a literal reading in fp64 (oracle/paged_ref.py): whole numbers, no tolerance."""
import numpy as np
import pytest
import torch

from oracle import paged_ref as P
from paged_cases import f, ints, normal


def test_oracle_on_a_worked_example():
    """Two channels tell three pages apart (d = 64, the others zero)."""
    bounds = np.zeros((3, 1, 2, 64))
    bounds[0, 0, :, 0] = [-1, 4]    # q+ = 2 on channel 0: 8
    bounds[1, 0, :, 1] = [-3, 9]    # q- = -1 on channel 1: 3
    bounds[2, 0, :, :2] = [[1, -2], [2, 5]]  # 4 + 2
    Q = np.zeros((1, 2, 64))
    Q[0, 0, 0], Q[0, 1, 1] = 2, -1  # two heads of one group
    table = np.array([[2, 1, 0, -1]])
    assert P.select(Q, bounds, table, 2, 16, [48], 0, 0).tolist() == [[[0, 2]]]      # scores 6, 3, 8
    assert P.select(Q, bounds, table, 1, 16, [48], 0, 0).tolist() == [[[2]]]
    assert P.select(Q, bounds, table, 2, 16, [33], 0, 1).tolist() == [[[0, 2]]]
    assert P.select(Q, bounds, table, 2, 16, [32], 0, 1).tolist() == [[[0, 1]]]
    assert P.select(Q, bounds, table, 3, 16, [64], 0, 1).tolist() == [[[0, 1, 2]]]   # the last page is missing
    assert P.select(Q, bounds, table, 4, 16, [0], 1, 1).tolist() == [[[-1] * 4]]


def run(B, Hq, Hk, R, d, lens, keep, first=1, recent=1, T=None, max_pages=None, seed=0, gone=0.0, change=None):
    from paper_2603_15619_amd import moda_page_select

    print("case", dict(B=B, Hq=Hq, Hk=Hk, R=R, d=d, lens=lens, keep=keep, first=first, recent=recent, seed=seed), flush=True)
    g = torch.Generator().manual_seed(seed)
    max_pages = max_pages or max([-(-n // R) for n in lens or [T]] + [1]) + 1
    n_pages = B * max_pages
    table = torch.randperm(n_pages, generator=g).view(B, max_pages).int()
    table[torch.rand((B, max_pages), generator=g) < gone] = -1
    x = normal(g, 2, n_pages, Hk, d)
    bounds = torch.stack([torch.minimum(x[0], x[1]), torch.maximum(x[0], x[1])], 2).contiguous()
    Q = normal(g, B, Hq, d)
    if change:
        change(Q, bounds, table)
    want = P.select(f(Q), f(bounds), table.numpy(), keep, R, lens, first, recent, T)
    out = torch.full((B, Hk, keep), -9, dtype=torch.int32, device="cuda")
    got = moda_page_select(Q.cuda(), bounds.cuda(), table.cuda(), keep, R, lengths=ints(lens), first=first, recent=recent, T=T, out=out)
    torch.cuda.synchronize()
    assert got is out
    assert np.array_equal(got.cpu().numpy(), want)
    return want


@pytest.mark.gpu
@pytest.mark.parametrize("c", [
    dict(B=1, Hq=1, Hk=1, R=16, d=64, lens=[1], keep=1, first=0, recent=0),
    dict(B=2, Hq=4, Hk=2, R=16, d=128, lens=[0, 33], keep=2),
    dict(B=3, Hq=6, Hk=2, R=32, d=64, lens=[1000, 999, 31], keep=7, gone=0.2),
    dict(B=2, Hq=16, Hk=1, R=64, d=128, lens=[8000, 5000], keep=10, first=2, recent=3),
    dict(B=1, Hq=3, Hk=3, R=16, d=64, lens=[5000], keep=100),
    dict(B=1, Hq=2, Hk=2, R=256, d=128, lens=[70000], keep=33, first=0, recent=1),
    dict(B=2, Hq=8, Hk=8, R=128, d=64, lens=[3000, 200], keep=64),          # more than there are
    dict(B=2, Hq=10, Hk=2, R=16, d=128, lens=None, T=513, keep=9),
    dict(B=3, Hq=4, Hk=4, R=16, d=64, lens=[700, -4, 600], T=640, max_pages=50, keep=5),  # below zero, above T
    dict(B=1, Hq=1, Hk=1, R=16, d=64, lens=[16 * 1100], keep=1100, gone=0.5),
    dict(B=1, Hq=1, Hk=1, R=16, d=64, lens=[16 * 1100], keep=1, first=1, recent=0),
    dict(B=1, Hq=2, Hk=1, R=16, d=128, lens=[16 * 9000 + 5], keep=400),
])
def test_select(c):
    run(**c, seed=len(str(c)))


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_equal_and_nearly_equal_scores(d):
    """Ties go to the lowest page; pages whose scores differ in the 40th bit are told apart."""
    def ties(Q, bounds, table):
        bounds[:] = bounds[:1]
    run(2, 4, 2, 16, d, [3000, 2000], 50, change=ties, seed=1)

    def near(Q, bounds, table):  # (one head: q of channel 5 is 1, of the last one 2^-30: the pages differ by multiples of 2^-37)
        bounds[:] = bounds[:1]
        Q.abs_()
        Q[:, :, 5], Q[:, :, -1] = 1.0, 2.0 ** -30
        bounds[:, :, 1, -1] = 1 + (torch.arange(bounds.shape[0])[:, None] * 37 % 128) / 128
    run(1, 2, 2, 16, d, [16 * 127], 20, change=near, seed=2)

    def groups(Q, bounds, table):  # four values only
        bounds[:] = bounds[torch.arange(bounds.shape[0]) % 4]
    run(1, 2, 2, 16, d, [16 * 2000], 777, change=groups, seed=3)


@pytest.mark.gpu
def test_infinities_and_nan():
    def some(Q, bounds, table):
        g = torch.Generator().manual_seed(5)
        n = bounds.shape[0]
        bounds[torch.rand(n, generator=g) < 0.1, :, 1, 3] = float("inf")
        bounds[torch.rand(n, generator=g) < 0.1, :, 0, 9] = float("-inf")
        bounds[torch.rand(n, generator=g) < 0.1, :, :, 20] = float("nan")
        Q[:, :, 3] = Q[:, :, 3].abs()
        Q[0, 0, 9] = 0.0
    run(2, 4, 2, 16, 64, [16 * 60, 16 * 90], 40, change=some, seed=1)

    def query(Q, bounds, table):
        Q[0, 1, 7] = float("nan")  # every page of its group counts alike
        Q[1, 2, 0] = float("inf")
    run(2, 4, 2, 16, 128, [16 * 60, 16 * 90], 20, change=query, seed=2)


@pytest.mark.gpu
def test_bounds_hold():
    """A page's score is at least the group's logits, summed, on any of its rows."""
    from paper_2603_15619_amd import moda_page_append, moda_page_select

    g = torch.Generator().manual_seed(8)
    Hk, G, R, d, n = 2, 4, 16, 64, 16 * 40
    K = normal(g, 1, Hk, n, d).cuda()
    pools = [torch.zeros((41, Hk, R, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    bounds = torch.zeros((41, Hk, 2, d), dtype=torch.bfloat16, device="cuda")
    table = ints(np.random.default_rng(0).permutation(41)[None, :40])
    moda_page_append(K, K, *pools, table, Kbounds=bounds)
    rows = K.view(1, Hk, 40, R, d)
    assert torch.equal(bounds[table[0].long()][:, :, 0], rows[0].amin(2).transpose(0, 1)) and torch.equal(bounds[table[0].long()][:, :, 1], rows[0].amax(2).transpose(0, 1))
    Q = normal(g, 1, G * Hk, d).cuda()
    Q[0, 0] = 8 * K[0, 0, 333]  # the first group's head 0 looks for row 333
    pages = moda_page_select(Q, bounds, table, 4, R, first=0, recent=0)
    assert 333 // R in pages[0, 0].tolist()
