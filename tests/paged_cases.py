"""Paged caches for the tests: pools, tables in a shuffled order, and their exact fp64 upcasts."""
import numpy as np
import torch

from paper_2603_15619_amd import synth

f = synth.to_f64


def ints(v, device="cuda"):
    return None if v is None else torch.tensor(np.asarray(v), dtype=torch.int32, device=device)


def values(codes, scales):
    """fp64 of a pool, from codes and scale bytes where it holds 8 bits."""
    x = codes.float().double().cpu().numpy()
    if scales is None:
        return x
    return x * np.repeat(2.0 ** (scales.cpu().numpy().astype(np.float64) - 127), 32, axis=-1)


def normal(g, *shape):
    return torch.randn(shape, generator=g).to(torch.bfloat16)


class Cache:
    """Pools on the device and, as .K, .V (fp64), what they hold.  lens: rows of each sequence; gone: (sequence, page)s without a page; spare pages
    hold NaN, and so do rows that no length covers."""

    def __init__(self, Hk, R, d, lens, max_pages=None, mx=False, seed=0, gone=(), change=None, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        need = [-(-max(n, 0) // R) for n in lens]
        self.max_pages = max(need + [1]) + 1 if max_pages is None else max_pages
        self.n_pages = sum(min(n, self.max_pages) for n in need) + 2
        order = torch.randperm(self.n_pages, generator=g).tolist()
        self.table = np.full((len(lens), self.max_pages), -1, dtype=np.int32)
        self.table[:, 1::2] = 1 << 30  # (no page either)
        used = np.zeros((self.n_pages, R), dtype=bool)
        for b, n in enumerate(lens):
            for p in range(min(need[b], self.max_pages)):
                page = order.pop()
                if (b, p) not in gone:
                    self.table[b, p] = page
                    used[page, :max(0, min(R, n - p * R))] = True
        self.Hk, self.R, self.d, self.lens, self.mx = Hk, R, d, lens, mx
        pools = [normal(g, self.n_pages, Hk, R, d) for _ in range(2)]
        if change:
            change(self, *pools)
        nan = ~torch.from_numpy(used)[:, None, :, None].expand(pools[0].shape)
        self.scales = [None, None]
        if mx:
            quantised = [plain_quantise(x) for x in pools]
            pools = [torch.where(nan, torch.full_like(q[0], 0x7f), q[0]).view(torch.float8_e4m3fn) for q in quantised]
            self.scales = [q[1].to(device) for q in quantised]
        else:
            pools = [torch.where(nan, torch.full_like(x, float("nan")), x) for x in pools]
        self.pools = [x.to(device) for x in pools]
        self.K, self.V = (values(x, s) for x, s in zip(self.pools, self.scales))

    def args(self):
        return dict(Kpages=self.pools[0], Vpages=self.pools[1], page_table=ints(self.table), Kscales=self.scales[0], Vscales=self.scales[1])


def plain_quantise(x):
    """bf16 -> (codes as uint8, scale bytes), by the library's own rounding to e4m3; finite values below 2^126."""
    y = x.double().unflatten(-1, (-1, 32))
    a = y.abs().amax(-1)
    mantissa, e = torch.frexp(a)
    e = torch.where(mantissa <= 0.875, e - 9, e - 8).clamp(min=-100)
    e = torch.where(a == 0, torch.full_like(e, -100), e)
    z = (y * torch.pow(torch.tensor(2.0, dtype=torch.float64), -e.double())[..., None]).float()
    return z.to(torch.float8_e4m3fn).view(torch.uint8).flatten(-2), (e + 127).to(torch.uint8)
