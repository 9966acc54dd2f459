"""The calls on a paged cache together, as a serving loop makes them; captured, at once, on views, far into large pools."""
import numpy as np
import pytest
import torch

from oracle import paged_ref as P
from paged_cases import f, ints, normal, values
from test_decode_paged import U, tolerances

pytestmark = pytest.mark.gpu


class Server:
    """A paged cache that grows; .ref: the same in fp64."""

    def __init__(self, B, Hk, R, d, n_pages, max_pages, mx, seed):
        self.g = torch.Generator().manual_seed(seed)
        self.B, self.Hk, self.R, self.d, self.mx = B, Hk, R, d, mx
        dt = torch.float8_e4m3fn if mx else torch.bfloat16
        self.pools = [torch.zeros((n_pages, Hk, R, d), dtype=torch.uint8 if mx else dt, device="cuda").view(dt) for _ in range(2)]
        self.scales = [torch.full((n_pages, Hk, R, d // 32), 127, dtype=torch.uint8, device="cuda") if mx else None for _ in range(2)]
        self.bounds = torch.zeros((n_pages, Hk, 2, d), dtype=torch.bfloat16, device="cuda")
        free = torch.randperm(n_pages, generator=self.g).tolist()
        self.table = np.array([[free.pop() for _ in range(max_pages)] for _ in range(B)], dtype=np.int32)
        self.lengths = ints([0] * B)
        self.ref = [np.zeros((n_pages, Hk, R, d)) for _ in range(2)] + [np.zeros((n_pages, Hk, 2, d))]

    def cache(self):
        return dict(Kpages=self.pools[0], Vpages=self.pools[1], page_table=ints(self.table), Kscales=self.scales[0], Vscales=self.scales[1])

    def append(self, counts, T):
        from paper_2603_15619_amd import moda_page_append

        K, V = normal(self.g, self.B, self.Hk, T, self.d), normal(self.g, self.B, self.Hk, T, self.d)
        self.lengths.add_(ints(counts))
        moda_page_append(K.cuda(), V.cuda(), **self.cache(), lengths=self.lengths, counts=ints(counts), Kbounds=self.bounds)
        P.append(f(K), f(V), *self.ref[:2], self.table, self.lengths.tolist(), counts, self.mx, self.ref[2])


@pytest.mark.parametrize("mx,G,R,d", [(False, 1, 16, 64), (True, 4, 16, 128), (False, 8, 32, 128), (True, 2, 64, 64)])
def test_serving_loop(mx, G, R, d):
    """Ragged prompts in two chunks, then tokens one by one; each attends all rows and the pages chosen for it.  Two sequences stop on the way,
    the oldest pages but the first go back when a sequence is long enough."""
    from paper_2603_15619_amd import moda_attn_decode_paged, moda_page_read, moda_page_select

    B, Hk, L = 4, 2, 3
    s = Server(B, Hk, R, d, 60 if R < 64 else 40, 9, mx, seed=R + G)
    s.append([70, 3, 40, 16], 70)
    s.append([5, 0, 33, 20], 40)
    for step in range(6):
        s.append([1, 1, 0 if step > 2 else 1, 1], 1)
        if step == 4 and R == 16:
            s.table[0, 1:3] = -1
        Q, Kd, Vd = normal(s.g, B, G * Hk, d), normal(s.g, B, Hk, L, d), normal(s.g, B, Hk, L, d)
        n = s.lengths.tolist()
        for x, sc, want in zip(s.pools, s.scales, s.ref):
            assert np.array_equal(values(x, sc), want)
        assert np.array_equal(f(s.bounds), s.ref[2])
        pages = moda_page_select(Q.cuda(), s.bounds, ints(s.table), 3, R, lengths=s.lengths)
        assert np.array_equal(pages.cpu().numpy(), P.select(f(Q), s.ref[2], s.table, 3, R, n))
        for chosen in (None, pages):
            O, LSE = moda_attn_decode_paged(Q.cuda(), **s.cache(), Kdepth=Kd.cuda(), Vdepth=Vd.cuda(), lengths=s.lengths, selected=chosen)
            r = P.decode(f(Q), *s.ref[:2], s.table, f(Kd), f(Vd), n, None if chosen is None else chosen.cpu().numpy())
            to, tl = tolerances(r, d)
            assert np.all(np.abs(f(O) - r["O"]) <= to) and np.all(np.abs(f(LSE) - r["LSE"]) <= tl)
        want = [np.zeros((B, Hk, 80, d)) for _ in range(2)]
        P.read(*s.ref[:2], s.table, *want, n, 7)
        for x, y in zip(moda_page_read(**s.cache(), lengths=s.lengths, first=7, T=80), want):
            assert np.array_equal(f(x), y)


@pytest.mark.parametrize("mx,G", [(False, 1), (True, 8)])
@pytest.mark.parametrize("wide", [False, True])
def test_captured_step(mx, G, wide):
    """One step of a loop as a graph, replayed as its lengths grow, with eager work and waits between: every replay gives what eager calls give.  Two
    graphs share a workspace."""
    from paper_2603_15619_amd import moda_attn_decode_paged, moda_page_append, moda_page_select

    B, Hk, R, d = 3, 2, 16, 128
    s = Server(B, Hk, R, d, 600 if wide else 60, 150 if wide else 16, mx, seed=G)
    s.append([200, 30, 7], 200)
    table, lengths = ints(s.table), s.lengths
    new = [torch.zeros((B, Hk, 1, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    Q = torch.zeros((B, G * Hk, d), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(32 << 20, dtype=torch.uint8, device="cuda")
    pages = torch.zeros((B, Hk, 4), dtype=torch.int32, device="cuda")
    outs = [(torch.zeros_like(Q), torch.zeros((B, G * Hk), device="cuda")) for _ in range(2)]
    pool = dict(Kpages=s.pools[0], Vpages=s.pools[1], page_table=table, Kscales=s.scales[0], Vscales=s.scales[1])

    def step(sparse, o):
        if not sparse:
            lengths.add_(1)
            moda_page_append(*new, **pool, lengths=lengths, Kbounds=s.bounds)
        else:
            moda_page_select(Q, s.bounds, table, 4, R, lengths=lengths, out=pages, workspace=ws)
        moda_attn_decode_paged(Q, **pool, lengths=lengths, selected=pages if sparse else None, out=o[0], lse=o[1], workspace=ws)

    state = [x.clone() for x in (lengths, s.bounds, *(p.view(torch.uint8) for p in s.pools))]
    step(False, outs[0])
    step(True, outs[1])  # (once before the capture)
    graphs = []
    for sparse in (False, True):
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(sparse, outs[int(sparse)])
        graphs.append(graph)
    lengths.copy_(state[0])
    s.bounds.copy_(state[1])
    for p, x in zip(s.pools, state[2:]):
        p.view(torch.uint8).copy_(x)
    for i in range(7):
        for x in new + [Q]:
            x.copy_(normal(s.g, *x.shape))
        before = [x.clone() for x in (lengths, s.bounds, *(p.view(torch.uint8) for p in s.pools), *(x for x in s.scales if x is not None))]
        for graph in graphs:
            graph.replay()
        if i % 2:
            torch.cuda.synchronize()
        got = [x.clone() for x in (*outs[0], *outs[1], pages, lengths, s.bounds, *(p.view(torch.uint8) for p in s.pools))]
        ws.random_(0, 256)  # (what a workspace holds is of no account)
        for x, y in zip((lengths, s.bounds, *(p.view(torch.uint8) for p in s.pools), *(x for x in s.scales if x is not None)), before):
            x.copy_(y)
        step(False, outs[0])
        step(True, outs[1])
        for x, y in zip(got, (*outs[0], *outs[1], pages, lengths, s.bounds, *(p.view(torch.uint8) for p in s.pools))):
            assert torch.equal(x, y), i


def test_calls_at_once_on_two_streams():
    """Workspaces of their own: each call gives what it gives alone, every time."""
    from paper_2603_15619_amd import moda_attn_decode_paged, moda_page_append, moda_page_read, moda_page_select

    def work(seed):
        s = Server(6, 2, 16, 64, 700, 100, bool(seed % 2), seed)
        s.append([1500, 40, 0, 700, 3, 900], 1500)
        Q, K = normal(s.g, 6, 16, 64).cuda(), normal(s.g, 6, 2, 9, 64).cuda()
        table, lens = ints(s.table), s.lengths

        def run():
            c = dict(s.cache(), Kpages=s.pools[0].clone(), Vpages=s.pools[1].clone(), page_table=table)
            b = s.bounds.clone()
            moda_page_append(K, K, **c, lengths=lens, Kbounds=b)
            pages = moda_page_select(Q, b, table, 20, 16, lengths=lens)
            r = [pages, b, *moda_attn_decode_paged(Q, **c, lengths=lens), *moda_attn_decode_paged(Q, **c, lengths=lens, selected=pages)]
            return r + list(moda_page_read(**c, lengths=lens, T=300))
        return run

    runs = [work(1), work(2)]
    alone = [r() for r in runs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    both = []
    for _ in range(3):
        for run, s in zip(runs, streams):
            with torch.cuda.stream(s):
                both.append(run())
    torch.cuda.synchronize()
    for i, got in enumerate(both):
        for x, y in zip(got, alone[i % 2]):
            assert torch.equal(x, y)


def test_tensors_inside_others():
    """Tables, lengths, counts and lists at any 4-byte address, the rest at any 16-byte one; other addresses are refused."""
    from paper_2603_15619_amd import MODAError, moda_attn_decode_paged, moda_page_append, moda_page_read, moda_page_select

    def inside(x, skip):  # a copy of x that starts `skip` elements into a larger tensor
        y = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
        big = torch.empty(y.numel() + skip, dtype=y.dtype, device=x.device)
        return big[skip:].view(y.shape).copy_(y).view(x.dtype)

    for mx in (False, True):
        s = Server(3, 2, 16, 64, 20, 5, mx, 3)
        s.append([60, 1, 33], 60)
        Q, K, table = normal(s.g, 3, 4, 64).cuda(), normal(s.g, 3, 2, 5, 64).cuda(), ints(s.table)
        unit = 16 if mx else 8
        a = dict(s.cache(), Kpages=s.pools[0].clone(), Vpages=s.pools[1].clone(), Kscales=s.scales[0].clone() if mx else None, Vscales=s.scales[1].clone() if mx else None)
        b = dict(Kpages=inside(s.pools[0], unit), Vpages=inside(s.pools[1], 3 * unit), page_table=inside(table, 1),
                 Kscales=inside(s.scales[0], 16) if mx else None, Vscales=inside(s.scales[1], 48) if mx else None)
        lens, counts, bounds = s.lengths, ints([5, 0, 2]), s.bounds.clone()
        bounds2 = inside(bounds, 8)
        moda_page_append(K, K, **a, lengths=lens, counts=counts, Kbounds=bounds)
        moda_page_append(inside(K, 8), inside(K, 24), **b, lengths=inside(lens, 3), counts=inside(counts, 1), Kbounds=bounds2)
        for n in a:
            if a[n] is not None:
                x, y = (t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t for t in (a[n], b[n]))
                assert torch.equal(x, y), n
        assert torch.equal(bounds, bounds2)
        pages = moda_page_select(Q, bounds, table, 3, 16, lengths=lens)
        assert torch.equal(pages, moda_page_select(inside(Q, 8), bounds2, b["page_table"], 3, 16, lengths=inside(lens, 1), out=inside(pages, 1)))
        want = moda_attn_decode_paged(Q, **a, lengths=lens, selected=pages)
        got = moda_attn_decode_paged(inside(Q, 16), **b, lengths=inside(lens, 1), selected=inside(pages, 3), out=inside(want[0], 8), lse=inside(want[1], 4))
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
        rows = moda_page_read(**a, lengths=lens, T=64)
        got = moda_page_read(**b, lengths=inside(lens, 1), out=tuple(inside(torch.zeros_like(x), 8) for x in rows))
        assert all(torch.equal(x, y) for x, y in zip(rows, got))
        for bad in (dict(a, Kpages=inside(s.pools[0], unit // 2)), dict(a, Vscales=inside(s.scales[1], 8)) if mx else dict(a, Vpages=inside(s.pools[1], 4))):
            for call in (lambda: moda_attn_decode_paged(Q, **bad), lambda: moda_page_read(**bad, T=4), lambda: moda_page_append(K, K, **bad)):
                with pytest.raises(MODAError, match="aligned"):
                    call()


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("G", [1, 8])
def test_pools_beyond_4_gib(G, mx):
    """Pages whose rows lie more than 2^32 bytes into their pools are written, chosen, attended and read back."""
    from paper_2603_15619_amd import moda_attn_decode_paged, moda_page_append, moda_page_read, moda_page_select

    d, R = 128, 256
    n_pages = ((1 << 32) // (R * d * (1 if mx else 2))) + 40
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GiB of device memory")
    dt = torch.uint8 if mx else torch.bfloat16
    pools = [torch.zeros((n_pages, 1, R, d), dtype=dt, device="cuda") for _ in range(2)]
    scales = [torch.zeros((n_pages, 1, R, d // 32), dtype=torch.uint8, device="cuda") if mx else None for _ in range(2)]
    if mx:
        pools = [x.view(torch.float8_e4m3fn) for x in pools]
    bounds = torch.zeros((n_pages, 1, 2, d), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(1)
    n = 3 * R + 100
    K, V, Q = normal(g, 2, 1, n, d), normal(g, 2, 1, n, d), normal(g, 2, G, d)
    table = np.array([[n_pages - 1, 5, n_pages - 30, n_pages - 2], [n_pages - 3, n_pages - 17, 0, n_pages - 20]], dtype=np.int32)
    c = dict(Kpages=pools[0], Vpages=pools[1], page_table=ints(table), Kscales=scales[0], Vscales=scales[1])
    moda_page_append(K.cuda(), V.cuda(), **c, Kbounds=bounds)
    held = [P.quantise(f(x))[0] if mx else f(x) for x in (K, V)]
    for x, want in zip(moda_page_read(**c, T=n, lengths=ints([n, n])), held):
        assert np.array_equal(f(x), want)
    # the oracle on a small pool of the same pages
    small = [np.zeros((8, 1, R, d)) for _ in range(2)]
    tiny = np.arange(8, dtype=np.int32).reshape(2, 4)
    for x, pool in zip(held, small):
        pool.reshape(2, 4 * R, d)[:, :n] = x[:, 0]
    b = bounds[torch.from_numpy(table).long().cuda().view(-1)]
    assert np.array_equal(f(b)[:3, 0, 0], small[0][:3, 0].min(1)) and np.array_equal(f(b)[3, 0, 1], small[0][3, 0, :100].max(0))
    pages = moda_page_select(Q.cuda(), bounds, ints(table), 3, R, lengths=ints([n, n - 200]))
    assert np.array_equal(pages.cpu().numpy(), P.select(f(Q), f(b), tiny, 3, R, [n, n - 200]))
    for chosen in (None, pages):
        O, LSE = moda_attn_decode_paged(Q.cuda(), **c, lengths=ints([n, n - 200]), selected=chosen)
        r = P.decode(f(Q), *small, tiny, lengths=[n, n - 200], selected=None if chosen is None else chosen.cpu().numpy())
        to, tl = tolerances(r, d)
        assert np.all(np.abs(f(O) - r["O"]) <= to) and np.all(np.abs(f(LSE) - r["LSE"]) <= tl)


def test_bounds_and_new_rows_beyond_4_gib():
    """Bounds of more than 2^32 bytes; new rows that lie more than 2^32 bytes into theirs."""
    from paper_2603_15619_amd import moda_page_append, moda_page_select

    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GiB of device memory")
    d = 128
    n = (1 << 32) // (4 * d) + 500
    bounds = torch.zeros((n, 1, 2, d), dtype=torch.bfloat16, device="cuda")
    table = ints([[n - 1 - 3 * i if i % 2 else i for i in range(40)]])
    bounds[n - 1 - 3 * 7, :, 1, 4] = 3.0
    bounds[n - 1 - 3 * 21, :, 1, 4] = 2.0
    bounds[8, :, 1, 4] = 1.0
    assert moda_page_select(torch.ones((1, 1, d), dtype=torch.bfloat16, device="cuda"), bounds, table, 3, 16, first=0, recent=0).tolist() == [[[7, 8, 21]]]
    del bounds
    T = (1 << 25) + 64  # 128 bytes a row
    K = torch.zeros((1, 1, T, 64), dtype=torch.bfloat16, device="cuda")
    K[0, 0, -1], K[0, 0, -70] = 5.0, 6.0
    pools = [torch.zeros((64, 1, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = torch.full((1, T // 16), -1, dtype=torch.int32, device="cuda")
    table[0, -8:] = torch.arange(8, dtype=torch.int32, device="cuda")
    moda_page_append(K, K, *pools, table)
    rows = pools[0][:8].view(-1, 64)
    assert rows[-1, 0] == 5.0 and rows[-70, 0] == 6.0 and rows.abs().sum() == 64 * 11 and torch.equal(pools[0], pools[1])


def test_like_prompt_attention():
    """The last token of a prompt: over the pages what the prompt's own attention gives for it."""
    from paper_2603_15619_amd import moda_attn_decode_paged, moda_attn_fwd, moda_page_append

    g = torch.Generator().manual_seed(6)
    B, Hq, Hk, T, d, L = 2, 8, 2, 333, 64, 3
    Q, K, V = (normal(g, B, h, T, d).cuda() for h in (Hq, Hk, Hk))
    Kd, Vd = (normal(g, B, Hk, T, L, d).cuda() for _ in range(2))
    O, LSE = moda_attn_fwd(Q, K, V, Kd, Vd)
    pools = [torch.empty((50, Hk, 16, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = ints(np.random.default_rng(0).permutation(50)[:42].reshape(2, 21))
    moda_page_append(K, V, *pools, table)
    o, lse = moda_attn_decode_paged(Q[:, :, -1].contiguous(), *pools, table, Kd[:, :, -1].contiguous(), Vd[:, :, -1].contiguous(), T=T)
    assert (o.float() - O[:, :, -1].float()).abs().max() <= 4 * U and (lse - LSE[:, :, -1]).abs().max() <= 1e-3
