"""Rows into the pages of a paged cache and back, against the definition in fp64 (oracle/paged_ref.py).

No tolerance: a row in bf16 pages is the row, an 8-bit row is the one rounding that the definition names, a bound is one of its values, and what
is read back is what is held.  The 8-bit numbers are off by what one rounding may be (test_quantisation_is_one_rounding)."""
import numpy as np
import pytest
import torch

from oracle import paged_ref as P
from paged_cases import Cache, f, ints, normal, values


def same(got, want):
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == want.shape and np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(np.nan_to_num(got), np.nan_to_num(want))


def test_oracle_quantise_on_known_values():
    x = np.zeros((7, 32))
    x[0, :4] = [448, 1, 0.0625 + 2.0 ** -7, -17]       # scale 1: 17 is halfway between 16 and 18, 16 has the even code
    x[1, :3] = [449, 2, 2.0 ** -9]                     # scale 2; 449 / 2 = 224.5 -> 224; 2^-10 of the scale is halfway to the least value
    x[2, 0] = 2.0 ** -120                              # below the least scale: rounds to nothing
    x[3, 0] = 2.0 ** 127 * 1.9921875                   # the largest bf16 number
    x[4, :2] = [np.inf, 1.75]
    x[5, :2] = [np.nan, -3.0 * 2.0 ** -6]
    v, e = P.quantise(x)
    assert e[:, 0].tolist() == [0, 1, -100, 120, -8, -13, -100]  # 1.75 = 448 * 2^-8; 3 * 2^-6 <= 448 * 2^-13 (= 3.5 * 2^-6)
    assert v[0, :4].tolist() == [448, 1, 0.0625 + 2.0 ** -7, -16]
    assert v[1, :3].tolist() == [448, 2, 0] and v[2, 0] == 0 and v[3, 0] == 1.875 * 2.0 ** 127
    assert np.isnan(v[4, 0]) and v[4, 1] == 1.75 and np.isnan(v[5, 0]) and v[5, 1] == -3.0 * 2.0 ** -6
    assert (P.E4M3[1:] > P.E4M3[:-1]).all() and P.E4M3[-1] == 448 and P.E4M3[1] == 2.0 ** -9


def test_oracle_quantise_against_the_library_rounding():
    from paged_cases import plain_quantise

    g = torch.Generator().manual_seed(1)
    x = normal(g, 500, 128) * torch.pow(2.0, torch.randint(-30, 30, (500, 128), generator=g).float()).bfloat16()
    codes, scales = plain_quantise(x)
    v, e = P.quantise(f(x))
    assert np.array_equal(v, values(codes.view(torch.float8_e4m3fn), scales)) and np.array_equal(e + 127, scales.numpy())


def test_quantisation_is_one_rounding():
    g = torch.Generator().manual_seed(2)
    x = f(normal(g, 2000, 64))
    v, e = P.quantise(x)
    unit = np.repeat(2.0 ** e, 32, axis=-1)
    assert np.all(np.abs(v - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * unit))
    assert np.array_equal(f(torch.from_numpy(v).to(torch.bfloat16)), v)  # bf16 holds what 8 bits stand for


def run_append(Hk, R, d, before, new, T, mx, counts=True, with_bounds=True, seed=0, change=None, capacity=None, lens=None):
    """Sequences of `before` rows grow by `new` of T padded rows."""
    from paper_2603_15619_amd import moda_page_append

    print("case", dict(Hk=Hk, R=R, d=d, before=before, new=new, T=T, mx=mx, seed=seed), flush=True)
    B = len(before)
    after = [a + n for a, n in zip(before, new)] if lens is None else lens
    c = Cache(Hk, R, d, after, capacity, mx, seed)
    g = torch.Generator().manual_seed(seed + 1)
    K, V = normal(g, B, Hk, T, d), normal(g, B, Hk, T, d)
    if change:
        change(K, V)
    bounds = normal(g, c.n_pages, Hk, 2, d) if with_bounds else None
    ref = [c.K.copy(), c.V.copy(), None if bounds is None else f(bounds)]
    old_codes = [x.view(torch.uint8).clone() for x in c.pools]
    written = P.append(f(K), f(V), *ref[:2], c.table, after, new if counts else None, mx, ref[2])
    bounds = None if bounds is None else bounds.cuda()
    r = moda_page_append(K.cuda(), V.cuda(), **c.args(), lengths=ints(after), counts=ints(new) if counts else None, Kbounds=bounds)
    torch.cuda.synchronize()
    assert r[0] is c.pools[0] and r[1] is c.pools[1]
    for x, s, want in zip(c.pools, c.scales, ref):
        same(values(x, s), want)
    if bounds is not None:
        same(f(bounds), ref[2])
    # nothing but the rows written has changed, to the bit
    rows = np.zeros((c.n_pages, R), dtype=bool)
    for page, slot in written:
        rows[page, slot] = True
    for x, old in zip(c.pools, old_codes):
        kept = x.view(torch.uint8)[torch.from_numpy(~rows).cuda()[:, None, :].expand(-1, Hk, -1)]
        assert torch.equal(kept, old[torch.from_numpy(~rows).cuda()[:, None, :].expand(-1, Hk, -1)])
    return c


APPENDS = [
    dict(Hk=1, R=16, d=64, before=[0], new=[1], T=1),
    dict(Hk=2, R=16, d=128, before=[5, 15, 16, 31], new=[1, 1, 1, 1], T=1),
    dict(Hk=3, R=32, d=64, before=[0, 31, 7, 100], new=[70, 0, 33, 1], T=70),
    dict(Hk=2, R=64, d=128, before=[0, 63, 64], new=[129, 2, 64], T=130),
    dict(Hk=1, R=128, d=64, before=[100, 0], new=[300, 1], T=300),
    dict(Hk=2, R=256, d=128, before=[0, 255, 200], new=[600, 3, 56], T=601),
    dict(Hk=5, R=16, d=128, before=[3, 9], new=[41, 2], T=50),
    dict(Hk=1, R=256, d=64, before=[250, 10], new=[7, 5], T=9),
]


@pytest.mark.gpu
@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("c", APPENDS)
def test_append(c, mx):
    run_append(**c, mx=mx, seed=len(str(c)))
    run_append(**c, mx=mx, seed=7, with_bounds=False)


@pytest.mark.gpu
@pytest.mark.parametrize("mx", [False, True])
def test_append_of_prompts_without_counts(mx):
    run_append(2, 32, 64, [0, 0, 0, 0], [100, 1, 64, 0], 100, mx, counts=False)


@pytest.mark.gpu
def test_append_with_odd_lengths_and_counts():
    """Counts below zero, above T and above the length; lengths below zero; rows that the table has no page for are left out."""
    from paper_2603_15619_amd import moda_page_append

    run_append(2, 16, 64, [0] * 5, [-3, 50, 9, 20, 1 << 30], 20, False, lens=[30, 40, 4, -7, 33])
    run_append(2, 16, 64, [0] * 3, [20, 20, 20], 20, True, lens=[70, 58, 1 << 30], capacity=4)  # 64 rows of capacity
    # a page in the middle is missing: its rows are dropped, the others written
    c = Cache(2, 16, 64, [50], gone=[(0, 1)])
    g = torch.Generator().manual_seed(3)
    K, V = normal(g, 1, 2, 50, 64), normal(g, 1, 2, 50, 64)
    ref = [c.K.copy(), c.V.copy()]
    assert len(P.append(f(K), f(V), *ref, c.table, [50])) == 34
    moda_page_append(K.cuda(), V.cuda(), **c.args(), lengths=ints([50]))
    same(values(c.pools[0], None), ref[0])
    same(values(c.pools[1], None), ref[1])


@pytest.mark.gpu
@pytest.mark.parametrize("mx", [False, True])
def test_append_of_extreme_values(mx):
    """Zeros, least and largest numbers, infinities and NaN with either sign, powers of two at the borders of a scale."""
    special = torch.tensor([0.0, -0.0, 1.0, 448.0, 449.0, -480.0, 2.0 ** -133, 3.3895e38, -3.3895e38, float("inf"), float("-inf"), float("nan"),
                            1.75, 1.7578125, 17.0, 19.0, -2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -92, 2.0 ** -110]).bfloat16()

    def change(K, V):
        g = torch.Generator().manual_seed(9)
        for x in (K, V):
            flat = x.view(-1, 32)
            pick = special[torch.randint(0, len(special), flat.shape, generator=g)]
            mode = torch.randint(0, 4, (flat.shape[0], 1), generator=g)
            one = torch.zeros_like(flat)
            one[:, 5] = pick[:, 5]
            sign = torch.where(torch.rand(flat.shape, generator=g) < 0.5, -1.0, 1.0).bfloat16()
            flat.copy_(torch.where(mode == 0, pick * sign, torch.where(mode == 1, one, torch.where(mode == 2, flat * pick[:, :1], flat))))
    run_append(2, 32, 128, [0, 20], [90, 40], 90, mx, change=change)


@pytest.mark.gpu
@pytest.mark.parametrize("Hk,R,d,lens,first,T,gone", [
    (1, 16, 64, [1], 0, 1, []), (2, 16, 128, [40, 0, 17], 0, 48, []), (3, 32, 64, [100, 99, 31], 30, 70, []),
    (2, 64, 128, [200, 64, 65], 63, 130, [(0, 1)]), (1, 128, 64, [500, 130], 127, 300, []), (2, 256, 128, [700, 3], 1, 900, [(0, 0)]),
    (2, 16, 64, [300], 299, 1, []), (2, 16, 128, [90], 93, 5, [])])
@pytest.mark.parametrize("mx", [False, True])
def test_read(Hk, R, d, lens, first, T, gone, mx):
    from paper_2603_15619_amd import moda_page_read

    c = Cache(Hk, R, d, lens, mx=mx, seed=T, gone=gone)
    out = [torch.full((len(lens), Hk, T, d), -7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ref = [f(x) for x in out]
    P.read(c.K, c.V, c.table, *ref, lens, first)
    r = moda_page_read(**c.args(), lengths=ints(lens), first=first, out=tuple(out))
    torch.cuda.synchronize()
    assert r[0] is out[0]
    for x, want in zip(out, ref):
        same(f(x), want)
    zeros = [np.zeros_like(x) for x in ref]
    P.read(c.K, c.V, c.table, *zeros, lens, first)
    for x, want in zip(moda_page_read(**c.args(), lengths=ints(lens), first=first, T=T), zeros):
        same(f(x), want)


@pytest.mark.gpu
def test_read_without_lengths_and_behind_the_table():
    from paper_2603_15619_amd import moda_page_read

    c = Cache(2, 16, 64, [48, 48], max_pages=3)
    K, V = moda_page_read(**c.args())
    assert K.shape == (2, 2, 48, 64)
    ref = [np.zeros((2, 2, 48, 64)) for _ in range(2)]
    P.read(c.K, c.V, c.table, *ref)
    same(f(K), ref[0])
    same(f(V), ref[1])
    K, _ = moda_page_read(**c.args(), lengths=ints([1 << 30, -5]), first=40, T=30)  # rows behind the table are not there
    ref = [np.zeros((2, 2, 30, 64)) for _ in range(2)]
    P.read(c.K, c.V, c.table, *ref, [1 << 30, -5], 40)
    same(f(K), ref[0])
    assert moda_page_read(**c.args(), first=48)[0].shape[2] == 0 and not moda_page_read(**c.args(), first=1 << 20, T=4)[0].any()


@pytest.mark.gpu
@pytest.mark.parametrize("mx", [False, True])
def test_what_was_appended_comes_back(mx):
    """Prompt, then single rows; pages of which two sequences share the first are read for both."""
    from paper_2603_15619_amd import moda_page_append, moda_page_read

    g = torch.Generator().manual_seed(4)
    B, Hk, R, d, n = 3, 2, 16, 128, 37
    dt = torch.float8_e4m3fn if mx else torch.bfloat16
    pools = [torch.zeros((20, Hk, R, d), dtype=torch.uint8 if mx else dt, device="cuda").view(dt) for _ in range(2)]
    scales = [torch.zeros((20, Hk, R, d // 32), dtype=torch.uint8, device="cuda") if mx else None for _ in range(2)]
    a = dict(Kpages=pools[0], Vpages=pools[1], page_table=ints([[3, 17, 0, 9], [5, 1, 2, 4], [11, 10, 19, 18]]), Kscales=scales[0], Vscales=scales[1])
    K, V = normal(g, B, Hk, n + 3, d).cuda(), normal(g, B, Hk, n + 3, d).cuda()
    moda_page_append(K[:, :, :n].contiguous(), V[:, :, :n].contiguous(), **a)
    lengths = ints([n] * B)
    for i in range(3):
        lengths.add_(1)
        moda_page_append(K[:, :, n + i:n + i + 1].contiguous(), V[:, :, n + i:n + i + 1].contiguous(), **a, lengths=lengths)
    for x, y in zip((K, V), moda_page_read(**a, lengths=lengths, T=n + 3)):
        same(f(y), P.quantise(f(x))[0] if mx else f(x))
    a["page_table"] = ints([[3, 17, 0, 9], [3, 1, 2, 4]])
    both = moda_page_read(**a, lengths=ints([16, 16]), T=16)[0]
    assert torch.equal(both[0], both[1])
