"""The softmax weights of the decoding step over pages: in 32 bits or nearly so for groups of up to four heads, as moda_attn_decode has them, rounded to
bf16 once for larger ones.

The measure is the error of the reference itself once it is rounded to bf16, e = ||bf16(ref) - ref||: what no bf16 output does without.  A call whose weights
are off by 2^-15 of themselves or less is off by e and nothing else that counts: their error, as random as the values, is 2^-15 / 2^-9 of e at most, and
32-bit logits, of size 10 and sums of 128 products, move a weight by 6e-5 at most, 0.03 of e: squares add up, so 1.001 e; 1.05 e is asked for.  Weights
rounded to bf16 add an error of about the size of e, so that the sum is 1.4 e; at most 2^-8 / sqrt(3) against e >= 2^-8 / sqrt(3) / 2, 2.3 e."""
import numpy as np
import pytest
import torch

from oracle import paged_ref as P
from paged_cases import Cache, f, ints, normal


def errors(G, Hk, R, d, lens, mx, L, seed, selected=None):
    from paper_2603_15619_amd import moda_attn_decode_paged

    c = Cache(Hk, R, d, lens, mx=mx, seed=seed)
    g = torch.Generator().manual_seed(seed + 100)
    Q = normal(g, len(lens), G * Hk, d)
    depth = [normal(g, len(lens), Hk, L, d) if L else None for _ in range(2)]
    O, _ = moda_attn_decode_paged(Q.cuda(), **c.args(), Kdepth=None if not L else depth[0].cuda(), Vdepth=None if not L else depth[1].cuda(),
                                  lengths=ints(lens), selected=ints(selected))
    r = P.decode(f(Q), np.nan_to_num(c.K), np.nan_to_num(c.V), c.table, *(None if x is None else f(x) for x in depth), lens, selected)["O"]
    rounded = f(torch.from_numpy(r).to(torch.bfloat16))
    return np.linalg.norm(f(O) - r) / np.linalg.norm(rounded - r)


@pytest.mark.gpu
@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 16, 24])
def test_error_beside_the_output_rounding(G, d, mx):
    for lens, L in (([300, 64, 1003, 517], 0), ([5000, 2048], 7), ([33000], 15)):
        e = errors(G, 4, 32, d, lens, mx, L, seed=G)
        print("case", dict(G=G, d=d, mx=mx, lens=lens), "%.3f of the rounding" % e, flush=True)
        assert e <= (1.05 if G <= 4 else 2.3)


@pytest.mark.gpu
@pytest.mark.parametrize("G", [1, 3, 4, 8, 20])
@pytest.mark.parametrize("n", [1, 16, 50, 3000])
def test_infinite_values(G, n):
    """An infinite value makes its channel infinite, in every head, and changes no other: also where a softmax weight is exactly 1."""
    from paper_2603_15619_amd import moda_attn_decode_paged

    c = Cache(1, 16, 64, [n, n])
    Q = normal(torch.Generator().manual_seed(0), 2, G, 64).cuda()
    O, LSE = moda_attn_decode_paged(Q, **c.args(), lengths=ints([n, n]))
    row = n - 1
    c.pools[1][c.table[1, row // 16], 0, row % 16, 9] = float("-inf")
    O2, LSE2 = moda_attn_decode_paged(Q, **c.args(), lengths=ints([n, n]))
    rest = np.delete(np.arange(64), 9)
    assert torch.equal(O[0], O2[0]) and torch.equal(LSE, LSE2) and torch.equal(O[1][:, rest], O2[1][:, rest])
    assert torch.isneginf(O2[1, :, 9]).all()
