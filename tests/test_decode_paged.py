"""The decoding step over a paged cache against fp64.

Tolerances: those of the step over contiguous caches (tests/test_decode_shared.py), whose sums are the same; 8-bit rows are exact numbers, so
that their quantisation does not enter."""
import numpy as np
import pytest
import torch

from oracle import paged_ref as P
from paged_cases import Cache, f, ints, normal

U = 2.0 ** -8


def tolerances(r, d):
    e = (d + 8) * 2.0 ** -24 * r["logit"]
    return 1.25 * U * (np.abs(r["O"]) + r["mag"]) + 1e-6, e + 5e-5 + 2.0 ** -21 * np.abs(np.where(np.isfinite(r["LSE"]), r["LSE"], 0))


def check(G, Hk, R, d, lens, L=0, La=None, mx=False, T=None, max_pages=None, selected=None, gone=(), seed=0, scale=None, scale_q=1.0, change=None,
          lengths=True, change_q=None, workspace=None):
    from paper_2603_15619_amd import moda_attn_decode_paged

    print("case", dict(G=G, Hk=Hk, R=R, d=d, lens=lens, L=L, mx=mx, T=T, seed=seed), flush=True)
    B, Hq, La = len(lens), G * Hk, L if La is None else La
    c = Cache(Hk, R, d, [min(n, T) if T is not None else n for n in lens], max_pages, mx, seed, gone, change)
    g = torch.Generator().manual_seed(seed + 100)
    Q = (normal(g, B, Hq, d) * scale_q).bfloat16()
    if change_q:
        change_q(Q)
    depth = [normal(g, B, Hk, La, d) if La else None for _ in range(2)]
    for x in depth:
        if x is not None:
            x[:, :, L:] = float("nan")
    K, V = np.nan_to_num(c.K, nan=0.0, posinf=np.inf, neginf=-np.inf) if change is None else c.K, c.V
    r = P.decode(f(Q), K, V, c.table, *(None if x is None else f(x) for x in depth), lens if lengths else None, selected, T, L, scale)
    out, lse = torch.full((B, Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.full((B, Hq), float("nan"), device="cuda")
    O, LSE = moda_attn_decode_paged(Q.cuda(), **c.args(), Kdepth=None if not La else depth[0].cuda(), Vdepth=None if not La else depth[1].cuda(),
                                    lengths=ints(lens) if lengths else None, selected=ints(selected), T=T, depth_count=L, scale=scale, out=out,
                                    lse=lse, workspace=workspace)
    torch.cuda.synchronize()
    to, tl = tolerances(r, d)
    finite = np.isfinite(r["LSE"])
    assert np.array_equal(finite, np.isfinite(f(LSE))) and np.all(f(LSE)[~finite] == -np.inf)
    eo, el = np.abs(f(O) - r["O"]) / to, np.abs(f(LSE)[finite] - r["LSE"][finite]) / tl[finite]
    print("   O %.3f LSE %.3f of the tolerance" % (eo.max(initial=0), el.max(initial=0)), flush=True)
    assert np.all(eo <= 1) and np.all(el <= 1)
    return O, LSE


CASES = [
    dict(G=1, Hk=1, R=16, d=64, lens=[1]),
    dict(G=1, Hk=2, R=16, d=128, lens=[40, 0, 16, 17], L=15, La=16),
    dict(G=2, Hk=2, R=32, d=64, lens=[33, 700, 31], L=1),
    dict(G=1, Hk=16, R=16, d=128, lens=[1003], L=15),
    dict(G=4, Hk=2, R=64, d=128, lens=[2000, 64, 65, 1], L=7),
    dict(G=3, Hk=1, R=128, d=64, lens=[1500, 0, 129]),
    dict(G=5, Hk=2, R=256, d=128, lens=[257, 900], L=31),
    dict(G=8, Hk=4, R=16, d=64, lens=[3000, 1, 2999], L=64, La=70),
    dict(G=16, Hk=1, R=32, d=128, lens=[5000, 33]),
    dict(G=33, Hk=2, R=16, d=64, lens=[300, 15], L=3),
    dict(G=80, Hk=1, R=64, d=128, lens=[400], L=100),
    dict(G=1, Hk=1, R=16, d=64, lens=[20011]),
    dict(G=8, Hk=1, R=256, d=128, lens=[40000]),
    dict(G=1, Hk=3, R=16, d=128, lens=[30000, 5]),
    dict(G=2, Hk=1, R=16, d=64, lens=[0, 0, 0], L=2),
    dict(G=4, Hk=1, R=32, d=128, lens=[0, 0]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("c", CASES)
def test_decode(c, mx):
    check(**c, mx=mx, seed=len(str(c)))


@pytest.mark.gpu
@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("G,d", [(1, 128), (4, 64), (16, 128)])
def test_many_sequences(G, d, mx):
    """More sequences than a wave has lanes; lengths from nothing to much."""
    rng = np.random.default_rng(G)
    lens = [int(2 ** x) - 1 for x in rng.uniform(0, 9, 150)]
    lens[3], lens[70], lens[149] = 0, 4000, 0
    check(G, 1, 16, d, lens, L=2, mx=mx, seed=G)


@pytest.mark.gpu
@pytest.mark.parametrize("B", [64, 65, 200, 256, 257, 1000, 1500])
@pytest.mark.parametrize("G,d,mx", [(1, 64, False), (8, 64, True)])
def test_batches_around_what_a_wave_looks_at(B, G, d, mx):
    """Short sequences, a few longer than one workgroup takes, empty ones at both ends; the table is wide, so that no sequence is known to be short."""
    lens = [(i * 37) % 50 for i in range(B)]
    lens[0], lens[1], lens[B // 2], lens[B - 2], lens[B - 1] = 0, 3000, 1300, 2100, 0
    check(G, 1, 16, d, lens, L=1, mx=mx, max_pages=200, seed=B)
    check(G, 1, 16, d, [0] * B, L=1, mx=mx, max_pages=200, seed=B)


@pytest.mark.gpu
@pytest.mark.parametrize("G", [1, 4, 12])
def test_lengths_out_of_range_and_bounds(G):
    check(G, 2, 16, 64, [100, -5, 1 << 30, 77], T=90, max_pages=7, L=3)   # below zero counts as zero, above T as T
    check(G, 2, 32, 128, [100, 100], lengths=False, T=100, max_pages=9)    # no lengths: all T
    check(G, 2, 16, 128, [0, 0], lengths=False, T=0, max_pages=2, L=4)
    check(G, 1, 16, 64, [50, 3], T=400, max_pages=2000)                    # a table much wider than the sequences


@pytest.mark.gpu
@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("G,R,d", [(1, 16, 128), (3, 32, 64), (16, 64, 128)])
def test_missing_pages(G, R, d, mx):
    """Pages given back at the front, in the middle, at the end, and all of them."""
    check(G, 2, R, d, [10 * R, 7 * R + 5, 2 * R, 3], gone=[(0, 0), (0, 1), (0, 5), (1, 7), (2, 0), (2, 1), (3, 0)], L=2, mx=mx)
    check(G, 2, R, d, [3 * R, 1], gone=[(0, 0), (0, 1), (0, 2), (1, 0)], mx=mx)


@pytest.mark.gpu
@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("G,R,d", [(1, 16, 64), (4, 64, 128), (8, 32, 64), (40, 16, 128)])
def test_selected_pages(G, R, d, mx):
    """Lists in any order, with -1 and pages that the sequence does not have among them, shorter than a wave and longer."""
    rng = np.random.default_rng(R)
    lens, Hk = [100 * R - 3, 5 * R, 1, 0], 2
    for n in (1, 7, 90):
        sel = np.full((4, Hk, n), -1, dtype=np.int32)
        for b, length in enumerate(lens):
            for g in range(Hk):
                pages = rng.permutation(max(1, -(-length // R)))[:n]
                sel[b, g, rng.permutation(n)[:len(pages)]] = pages
        sel[2, 0, 0] = 1 << 30
        check(G, Hk, R, d, lens, L=3, mx=mx, selected=sel, gone=[(0, 4), (1, 0)], seed=n)
    check(G, Hk, R, d, lens, mx=mx, selected=np.full((4, Hk, 5), -1, dtype=np.int32))


@pytest.mark.gpu
@pytest.mark.parametrize("G", [1, 2, 8])
def test_scales_and_large_logits(G):
    check(G, 1, 16, 64, [1000, 33], L=4, scale=1.0, scale_q=3.0)
    check(G, 1, 32, 128, [3000], L=4, mx=True, scale=0.7, scale_q=2.0)


@pytest.mark.gpu
@pytest.mark.parametrize("G", [1, 4, 16])
def test_lowest_and_infinite_logits(G):
    """Keys that make logits of -inf weigh nothing, also where a sequence has no others; large negative ones are ordinary."""
    def rows(c, K, V):
        K[:, :, ::3, 0] = float("-inf")
    check(G, 1, 16, 64, [100, 16], change=rows, change_q=lambda Q: Q[:, :, 0].fill_(1.0))

    def all_rows(c, K, V):
        K[:, :, :, 0] = float("-inf")
    O, LSE = check(G, 1, 16, 128, [40, 17], change=all_rows, change_q=lambda Q: Q[:, :, 0].fill_(1.0))
    assert not O.any() and torch.isneginf(LSE).all()

    def low(c, K, V):
        K[:, :, :, 0] = -3e38
    check(G, 1, 16, 64, [40, 17], change=low, change_q=lambda Q: Q[:, :, 0].fill_(1.0), scale=1e-36)


@pytest.mark.gpu
@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("G", [1, 4, 16])
def test_nan_reaches_its_own_sequence_only(G, mx):
    from paper_2603_15619_amd import moda_attn_decode_paged

    c = Cache(1, 16, 64, [60, 60, 60, 60], mx=mx)
    Q = normal(torch.Generator().manual_seed(0), 4, G, 64).cuda()
    O, LSE = moda_attn_decode_paged(Q, **c.args(), lengths=ints([60] * 4))
    for pool, at in zip(c.pools, ((c.table[1, 2], 0, 3, 7), (c.table[2, 0], 0, 1, 9))):
        if mx:
            pool.view(torch.uint8)[at] = 0x7f
        else:
            pool[at] = float("nan")
    O2, LSE2 = moda_attn_decode_paged(Q, **c.args(), lengths=ints([60] * 4))
    assert torch.equal(O[0], O2[0]) and torch.equal(O[3], O2[3]) and torch.equal(LSE[[0, 2, 3]], LSE2[[0, 2, 3]])
    assert O2[1].isnan().all() and LSE2[1].isnan().all()
    assert O2[2, :, 9].isnan().all() and torch.equal(O2[2, :, :9], O[2, :, :9]) and torch.equal(O2[2, :, 10:], O[2, :, 10:])


@pytest.mark.gpu
def test_like_the_step_over_contiguous_caches():
    """The same rows in pages and in one array: the results of both calls lie within the tolerance of each other's definition."""
    from paper_2603_15619_amd import moda_attn_decode_paged, moda_attn_decode_shared, moda_page_read

    for G, d in ((1, 128), (4, 64), (16, 128)):
        lens = [700, 33, 512]
        c = Cache(2, 64, d, lens)
        K, V = moda_page_read(**c.args(), lengths=ints(lens))
        Q = normal(torch.Generator().manual_seed(1), 3, 2 * G, d).cuda()
        a, b = moda_attn_decode_paged(Q, **c.args(), lengths=ints(lens)), moda_attn_decode_shared(Q, None, None, K, V, lengths=ints(lens))
        assert (a[0].float() - b[0].float()).abs().max() <= 4 * U and (a[1] - b[1]).abs().max() <= 1e-4


@pytest.mark.gpu
def test_workspace_does_not_depend_on_the_lengths():
    import ctypes

    from paper_2603_15619_amd.binding import MODAPages, MODAShape, lib

    sizes = set()
    for T, max_pages in ((1, 1), (16, 4), (60000, 4000), (1 << 20, 1 << 16)):
        x, s = MODAPages(100, 16, max_pages, 0), MODAShape(3, 8, 2, T, 64, 0, 0, 1, 0.0, 1)
        sizes.add(lib().moda_attn_decode_paged_workspace_bytes(ctypes.byref(x), ctypes.byref(s)))
    assert len(sizes) == 1 and sizes.pop() > 0
    # a workspace of exactly that size, between guards
    lens = [5000, 3, 800]
    x, s = MODAPages(100, 16, 400, 0), MODAShape(3, 8, 2, 1, 64, 0, 0, 1, 0.0, 1)
    n = lib().moda_attn_decode_paged_workspace_bytes(ctypes.byref(x), ctypes.byref(s))
    ws = torch.full((n + 8192,), 0x5a, dtype=torch.uint8, device="cuda")
    check(4, 2, 16, 64, lens, workspace=ws[4096:4096 + n])
    assert (ws[:4096] == 0x5a).all() and (ws[4096 + n:] == 0x5a).all()
