"""8-bit pages bit by bit: the codes and scale bytes that an append writes are those of the library's own rounding to e4m3, zeros with
their sign among them (fp64 values, which the tests of tests/test_page_rows.py compare, do not tell the zeros apart)."""
import pytest
import torch

from paged_cases import normal, plain_quantise


def signed_rows(g, *shape):
    """Rows of N(0,1) with zeros of both signs, values that the scale of their block rounds to a zero, and blocks of nothing else."""
    x = normal(g, *shape)
    flat = x.view(-1, 32)
    sign = torch.where(torch.rand(flat.shape, generator=g) < 0.5, -1.0, 1.0).bfloat16()
    small = torch.tensor([0.0, 2.0 ** -12, 2.0 ** -20, 2.0 ** -60, 2.0 ** -133]).bfloat16()[torch.randint(0, 5, flat.shape, generator=g)]
    flat.copy_(torch.where(torch.rand(flat.shape, generator=g) < 0.5, small * sign, flat))
    flat[::5] = small[::5] * sign[::5]
    flat[1::5, 7] = 2.0 ** 100  # next to it 2^-60 underflows in 32 bits already
    flat[2::5] = 0.0 * sign[2::5]
    return x


def test_rows_hold_what_they_say():
    x = signed_rows(torch.Generator().manual_seed(0), 1, 2, 60, 64)
    codes, _ = plain_quantise(x)
    assert (codes == 0x80).sum() > 500 and (codes == 0).sum() > 500
    assert torch.equal(codes >> 7, x.signbit().to(torch.uint8))  # a rounding keeps the sign


@pytest.mark.gpu
@pytest.mark.parametrize("R,d", [(16, 64), (64, 128)])
def test_codes_and_signs_of_zeros(R, d):
    from paper_2603_15619_amd import moda_page_append, moda_page_read

    g = torch.Generator().manual_seed(R)
    B, Hk, T = 2, 2, 77
    K, V = signed_rows(g, B, Hk, T, d), signed_rows(g, B, Hk, T, d)
    n = -(-T // R)
    pools = [torch.full((B * n, Hk, R, d), 0x33, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
    scales = [torch.full((B * n, Hk, R, d // 32), 0x44, dtype=torch.uint8, device="cuda") for _ in range(2)]
    bounds = torch.zeros((B * n, Hk, 2, d), dtype=torch.bfloat16, device="cuda")
    table = torch.arange(B * n, dtype=torch.int32, device="cuda").view(B, n)
    c = dict(Kpages=pools[0], Vpages=pools[1], page_table=table, Kscales=scales[0], Vscales=scales[1])
    moda_page_append(K.cuda(), V.cuda(), **c, Kbounds=bounds)
    back = moda_page_read(**c, lengths=torch.full((B,), T, dtype=torch.int32, device="cuda"), T=T)
    torch.cuda.synchronize()

    def rows(x):  # [B, Hk, T, ...]
        return x.cpu().view(B, n, Hk, R, -1).transpose(1, 2).reshape(B, Hk, n * R, -1)[:, :, :T]
    for x, pool, scale, y in zip((K, V), pools, scales, back):
        codes, bytes_ = plain_quantise(x)
        assert torch.equal(rows(scale), bytes_)
        got = rows(pool.view(torch.uint8))
        bad = got != codes
        assert not bad.any(), "%d codes differ, first %#x for %#x" % (bad.sum(), got[bad][0], codes[bad][0])
        assert torch.equal(y.cpu().signbit(), x.signbit())
