"""The decoding step over pages of long caches: how far its outputs are off as a whole, and the cut of many rows into slices.

The bound on single elements (tests/test_decode_paged.py) is one of sum(w |v|), which long sequences of N(0,1) rows do not make smaller while their
outputs shrink with the root of their length.  So the outputs of a (sequence, key/value head) are compared as a vector too, ||O - ref|| / ||ref||.
O's own rounding to bf16 is off by 2^-8 of a value at most and, evenly spread over a step, by 2^-8 / sqrt(3) in the root mean square.  Groups of five
heads and more round every softmax weight to bf16 too: sum(w e v) with e as spread as that is to sum(w v), v random, as e is to 1.  Together
sqrt(1/3 + 1/3) 2^-8, and half as much again, more than four deviations of the norm of 64 numbers: 0.0048; without rounded weights 2^-8 itself.  32-bit
sums add 2^-24 times the logits' size and the like: nothing beside it.  A page of 256 rows that is lost among n changes O by sqrt(256 / n) of it: 0.08 of 40000 rows.
"""
import ctypes

import numpy as np
import pytest
import torch

from oracle import paged_ref as P
from paged_cases import Cache, f, ints, normal
from test_decode_paged import tolerances

U = 2.0 ** -8


def norm_bound(G):
    return U if G <= 4 else 1.5 * (2 / 3) ** 0.5 * U


def off(O, ref, Hk):
    """[B, Hk]: ||O - ref|| / ||ref||, 0 where ref is 0."""
    B = ref.shape[0]
    e, n = (np.linalg.norm(x.reshape(B, Hk, -1), axis=-1) for x in (O - ref, ref))
    return np.where(n > 0, e / np.where(n > 0, n, 1), 0.0)


def compare(O, LSE, r, G, Hk, d):
    to, tl = tolerances(r, d)
    finite = np.isfinite(r["LSE"])
    assert np.array_equal(finite, np.isfinite(f(LSE)))
    e, eo, el = off(f(O), r["O"], Hk), np.abs(f(O) - r["O"]) / to, np.abs(f(LSE)[finite] - r["LSE"][finite]) / tl[finite]
    print("   norm %.3f, O %.3f, LSE %.3f of the bounds" % (e.max() / norm_bound(G), eo.max(), el.max(initial=0)), flush=True)
    assert np.all(e <= norm_bound(G)) and np.all(eo <= 1) and np.all(el <= 1)


def workspace_bytes(c, B, Hq, Hk, d, T):
    from paper_2603_15619_amd.binding import MODAPages, MODAShape, lib

    x, s = MODAPages(c.n_pages, c.R, c.max_pages, int(c.mx)), MODAShape(B, Hq, Hk, T, d, 0, 0, 1, 0.0, 1)
    return lib().moda_attn_decode_paged_workspace_bytes(ctypes.byref(x), ctypes.byref(s))


def run(G, Hk, R, d, lens, L=0, mx=False, seed=0, max_pages=None):
    """In a workspace of just the size that is asked for, between guards."""
    from paper_2603_15619_amd import moda_attn_decode_paged

    print("case", dict(G=G, Hk=Hk, R=R, d=d, lens=lens[:8], B=len(lens), L=L, mx=mx, seed=seed), flush=True)
    B = len(lens)
    c = Cache(Hk, R, d, lens, max_pages, mx, seed)
    g = torch.Generator().manual_seed(seed + 100)
    Q = normal(g, B, G * Hk, d)
    depth = [normal(g, B, Hk, L, d) if L else None for _ in range(2)]
    r = P.decode(f(Q), np.nan_to_num(c.K), np.nan_to_num(c.V), c.table, *(None if x is None else f(x) for x in depth), lens)
    n = workspace_bytes(c, B, G * Hk, Hk, d, c.max_pages * R)
    ws = torch.full((n + 8192,), 0x5a, dtype=torch.uint8, device="cuda")
    O, LSE = moda_attn_decode_paged(Q.cuda(), **c.args(), Kdepth=None if not L else depth[0].cuda(), Vdepth=None if not L else depth[1].cuda(),
                                    lengths=ints(lens), workspace=ws[4096:4096 + n])
    torch.cuda.synchronize()
    assert (ws[:4096] == 0x5a).all() and (ws[4096 + n:] == 0x5a).all()
    compare(O, LSE, r, G, Hk, d)


@pytest.mark.gpu
@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 8, 16, 17, 32, 40])
def test_outputs_as_vectors(G, d, mx):
    run(G, 2, 16, d, [64, 200, 1003], mx=mx, seed=G)
    run(G, 1, 64, d, [6000, 777, 2049], L=15, mx=mx, seed=G)
    run(G, 1, 256, d, [40000], L=1, mx=mx, seed=G)


@pytest.mark.gpu
@pytest.mark.parametrize("G,d,mx", [(1, 64, False), (8, 64, False), (1, 128, True), (20, 64, True)])
def test_lengths_about_powers_of_two(G, d, mx):
    run(G, 1, 64, d, [65535, 65536, 65537, 1], mx=mx, seed=G)
    run(G, 1, 128, d, [131071, 3, 131073], L=2, mx=mx, seed=G)


@pytest.mark.gpu
@pytest.mark.parametrize("G,d,mx", [(1, 64, False), (2, 128, True), (8, 64, True), (20, 64, False)])
def test_many_sequences_with_a_long_one_among_them(G, d, mx):
    """More sequences than a wave looks at: their slices are dealt out by a kernel of its own."""
    lens = [(i * 37) % 90 for i in range(300)]
    lens[0], lens[1], lens[150], lens[298], lens[299] = 0, 70000, 66000, 9000, 0
    run(G, 1, 64, d, lens, mx=mx, seed=G, max_pages=1100)


class Repeated:
    """Long sequences whose tables name the pages of a small pool over and over; the reference counts each page as often as it is named."""

    def __init__(self, B, Hk, R, d, lens, n_pages, mx, seed, device="cuda"):
        self.c = Cache(Hk, R, d, [n_pages * R], mx=mx, seed=seed, device=device)
        self.lens, self.max_pages = lens, max(-(-n // R) for n in lens) + 3
        self.n_pages, self.R, self.mx = self.c.n_pages, R, mx
        rng = np.random.default_rng(seed)
        held = self.c.table[0, :n_pages]
        self.table = held[rng.integers(0, n_pages, (B, self.max_pages))].astype(np.int32)

    def args(self):
        return dict(self.c.args(), page_table=ints(self.table))

    def decode(self, Q, R):
        B, Hq, d = Q.shape
        Hk = self.c.Hk
        G = Hq // Hk
        r = {"O": np.zeros((B, Hq, d)), "LSE": np.zeros((B, Hq)), "mag": np.zeros((B, Hq, d)), "logit": np.zeros((B, Hq))}
        K, V = np.nan_to_num(self.c.K), np.nan_to_num(self.c.V)
        for b, n in enumerate(self.lens):
            times = np.zeros((self.n_pages, R))
            np.add.at(times, self.table[b, :n // R], np.ones(R))
            if n % R:
                times[self.table[b, n // R], :n % R] += 1
            for g in range(Hk):
                k, v, t = K[:, g].reshape(-1, d), V[:, g].reshape(-1, d), times.reshape(-1)
                s = Q[b, g * G:g * G + G] @ k.T * d ** -0.5
                m = s[:, t > 0].max(1, keepdims=True)
                e = np.exp(s - m) * t
                z = e.sum(1, keepdims=True)
                h = slice(g * G, g * G + G)
                r["O"][b, h], r["mag"][b, h], r["LSE"][b, h] = e / z @ v, e / z @ np.abs(v), (m + np.log(z))[:, 0]
                r["logit"][b, h] = d ** -0.5 * (np.abs(Q[b, h]) @ np.abs(k).T).max(1)
        return r


def test_reference_of_repeated_pages_is_the_oracle():
    x = Repeated(2, 2, 16, 64, [100, 333], 5, False, 0, "cpu")
    Q = f(normal(torch.Generator().manual_seed(0), 2, 4, 64))
    got, want = x.decode(Q, 16), P.decode(Q, np.nan_to_num(x.c.K), np.nan_to_num(x.c.V), x.table, lengths=x.lens)
    for n in ("O", "LSE", "mag"):
        assert np.allclose(got[n], want[n], rtol=1e-12, atol=1e-14)
    assert np.all(got["logit"] >= want["logit"])


@pytest.mark.gpu
@pytest.mark.parametrize("G,Hk,d,mx,lens", [
    (8, 2, 64, False, [700001, 300000]),             # slices of the least size that several rounds have (2048 rows)
    (4, 4, 64, True, [900000, 1, 800077]),           # ... of more than that
    (24, 1, 128, False, [1 << 21]),
    (1, 2, 64, False, [600001, 5]),                  # vector ALUs: more than 512 rows
    (2, 1, 128, True, [1 << 21, 70000]),
])
def test_slices_in_several_rounds(G, Hk, d, mx, lens):
    from paper_2603_15619_amd import moda_attn_decode_paged

    print("case", dict(G=G, Hk=Hk, d=d, mx=mx, lens=lens), flush=True)
    B, R = len(lens), 64
    x = Repeated(B, Hk, R, d, lens, 600, mx, G)
    Q = normal(torch.Generator().manual_seed(G), B, G * Hk, d)
    n = workspace_bytes(x, B, G * Hk, Hk, d, x.max_pages * R)
    ws = torch.full((n + 8192,), 0x5a, dtype=torch.uint8, device="cuda")
    O, LSE = moda_attn_decode_paged(Q.cuda(), **x.args(), lengths=ints(lens), workspace=ws[4096:4096 + n])
    torch.cuda.synchronize()
    assert (ws[:4096] == 0x5a).all() and (ws[4096 + n:] == 0x5a).all()
    compare(O, LSE, x.decode(f(Q), R), G, Hk, d)


@pytest.mark.gpu
@pytest.mark.parametrize("G", [1, 8])
def test_captured_step_of_many_sequences(G):
    """300 sequences, whose slices a kernel of its own deals out, as a graph: replayed as they grow, over workspaces of any content."""
    from paper_2603_15619_amd import moda_attn_decode_paged

    lens = [(i * 53) % 200 for i in range(300)]
    lens[7], lens[299] = 5000, 1700
    c = Cache(1, 16, 64, [n + 64 for n in lens], max_pages=400, seed=G)
    Q = normal(torch.Generator().manual_seed(G), 300, G, 64).cuda()
    lengths, a = ints(lens), c.args()
    ws = torch.empty(workspace_bytes(c, 300, G, 1, 64, 6400), dtype=torch.uint8, device="cuda")
    O, LSE = torch.zeros_like(Q), torch.zeros((300, G), device="cuda")
    step = lambda: moda_attn_decode_paged(Q, **a, lengths=lengths, out=O, lse=LSE, workspace=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(6):
        lengths.add_(ints([(b * 7 + i) % 10 for b in range(300)]))
        ws.random_(0, 256)
        graph.replay()
        if i % 2:
            torch.cuda.synchronize()
        got = O.clone(), LSE.clone()
        ws.random_(0, 256)
        step()
        assert torch.equal(got[0], O) and torch.equal(got[1], LSE), i
    r = P.decode(f(Q), np.nan_to_num(c.K), np.nan_to_num(c.V), c.table, lengths=lengths.tolist())
    to, tl = tolerances(r, 64)
    finite = np.isfinite(r["LSE"])
    assert np.all(np.abs(f(O) - r["O"]) <= to) and np.all(np.abs(f(LSE)[finite] - r["LSE"][finite]) <= tl[finite]) and np.isneginf(f(LSE)[~finite]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("G,d", [(1, 128), (4, 64), (16, 128)])
def test_like_contiguous_caches_as_vectors(G, d):
    """The same rows in pages and in one array: apart by what both calls may be off."""
    from paper_2603_15619_amd import moda_attn_decode_paged, moda_attn_decode_shared, moda_page_read

    lens = [700, 133, 5120]
    c = Cache(2, 64, d, lens)
    K, V = moda_page_read(**c.args(), lengths=ints(lens))
    Q = normal(torch.Generator().manual_seed(1), 3, 2 * G, d).cuda()
    a, b = moda_attn_decode_paged(Q, **c.args(), lengths=ints(lens)), moda_attn_decode_shared(Q, None, None, K, V, lengths=ints(lens))
    assert np.all(off(f(a[0]), f(b[0]), 2) <= 2 * norm_bound(G))


# ---------------------------------------------------------------- the arithmetic of the cut, on the host
def slices(lens, units, least, good):
    """How many slices each sequence has: the cut's definition, as moda_decode_paged.hip has it."""
    total = sum(lens)

    def share(workgroups):
        n = -(-total * units // workgroups)
        return -(-n // least) * least
    per = min(max(min(share(256), max(share(512), 512), max(share(2048), good)), least), 1 << 30)
    return [max(-(-n // per), 1) for n in lens]


def test_workspace_has_room_for_every_slice():
    """The library's workspace, which it sizes without the lengths, has a state for every slice of any lengths."""
    from paper_2603_15619_amd.binding import MODAPages, MODAShape, lib

    rng = np.random.default_rng(0)
    closest = 1 << 30
    for i in range(4000):
        d, mx = int(rng.choice([64, 128])), bool(rng.integers(2))
        G, Hk, B = int(rng.choice([1, 2, 3, 8, 16, 17, 32, 33, 70])), int(rng.choice([1, 2, 3, 8, 16, 40])), int(2 ** rng.uniform(0, 11))
        heads = G if G <= 2 else 16 if G <= 16 else 32
        units = Hk * -(-G // heads)
        least = 4 * 4 * 64 * (16 if mx else 8) // d if G <= 2 else 128
        top = 2.0 ** rng.uniform(0, 30)
        lens = [int(top * u) for u in rng.random(B) ** rng.choice([0.1, 1, 10])]
        if i % 5 == 0:  # a total just behind or at a multiple of what the workgroups share
            k = int(rng.choice([256, 512, 2048])) * least
            lens[0] += (-sum(lens)) % k + int(rng.integers(-1, 2))
            lens[0] = min(max(lens[0], 0), 1 << 30)
        x, s = MODAPages(100, 256, 1 << 22, int(mx)), MODAShape(B, G * Hk, Hk, 1 << 30, d, 0, 0, 1, 0.0, 1)
        n = lib().moda_attn_decode_paged_workspace_bytes(ctypes.byref(x), ctypes.byref(s))
        states, rest = divmod(n - 8 * B, 4 * G * Hk * (d + 2))
        assert rest == 0
        used = sum(slices(lens, units, least, 512 if G <= 2 else 2048))
        assert used <= states, (lens, G, Hk, d, mx)
        closest = min(closest, states - used)
    assert closest == 0  # (and no more than it needs)
