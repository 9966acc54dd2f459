"""Eviction from a sequence cache (moda_cache_evict): bits are moved, so everything is compared exactly."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import cache_ref as R


def cache(B, Hk, T, d, dtype, seed, kind="floats", shuffled=False, kv_alloc=None):
    kv_alloc = kv_alloc or T
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    K, V = (torch.randn((B, Hk, kv_alloc, d), generator=g).to(dt).cuda() for _ in range(2))
    W = torch.rand((B, Hk, kv_alloc), generator=g)
    if kind == "ties":
        W = (W * 4).floor()
    elif kind == "zeros":
        W = torch.zeros_like(W)
    elif kind == "mixed":
        odd = torch.tensor([float("inf"), float("-inf"), float("nan"), -0.0, 0.0, -1.5, 1e-45, 3e38])
        pick = torch.randint(0, 16, W.shape, generator=g)
        W = torch.where(pick < 8, odd[pick.clamp(max=7)], W)
    pos = torch.arange(kv_alloc).expand(B, Hk, kv_alloc)
    if shuffled:
        pos = torch.stack([torch.stack([torch.randperm(kv_alloc, generator=g) for _ in range(Hk)]) for _ in range(B)]) * 2 + 5
    return K, V, W.cuda(), pos.int().contiguous().cuda()


def check(B, Hk, T, d, keep, recent, dtype="bf16", lens=None, kind="floats", shuffled=False, positions=True, in_place=False,
          kv_alloc=None, out_alloc=None, seed=0):
    from paper_2603_15619_amd import moda_cache_evict

    print("case", dict(B=B, Hk=Hk, T=T, d=d, keep=keep, recent=recent, dtype=dtype, lens=lens, kind=kind, in_place=in_place), flush=True)
    K, V, W, pos = cache(B, Hk, T, d, dtype, seed, kind, shuffled, kv_alloc)
    if not positions:
        pos = None
    before = [None if x is None else x.clone() for x in (K, V, W, pos)]
    lengths = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    n = min(keep, T)
    out = None
    if not in_place:
        rows = out_alloc or n
        out = (torch.full((B, Hk, rows, d), 9.0, dtype=K.dtype, device="cuda"), torch.full((B, Hk, rows, d), 9.0, dtype=K.dtype, device="cuda"),
               torch.full((B, Hk, rows), 9.0, device="cuda"), None if pos is None else torch.full((B, Hk, rows), 9, dtype=torch.int32, device="cuda"))
    index, new = moda_cache_evict(K, V, W, keep, recent, pos, lengths, T, out)
    torch.cuda.synchronize()
    want, want_len = R.evict_index(before[2].double().cpu().numpy(), keep, recent, None if pos is None else before[3].cpu().numpy(), lens, T)
    assert np.array_equal(index.cpu().numpy(), want) and np.array_equal(new.cpu().numpy(), want_len)
    if lens is not None and in_place:
        assert new is lengths
    at = torch.from_numpy(want).cuda().long()
    live = at >= 0
    for got, old in zip(out or (K, V, W, pos), before):
        if old is None:
            continue
        rest = old if in_place else torch.full_like(got, 9)
        moved = old.gather(2, at.clamp(min=0)[..., None].expand(*at.shape, d)) if old.dim() == 4 else old.gather(2, at.clamp(min=0))
        exp = rest.clone()
        exp[:, :, :n] = torch.where(live[..., None] if old.dim() == 4 else live, moved, rest[:, :, :n])
        bits = lambda x: x.contiguous().view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32)
        assert torch.equal(bits(got), bits(exp))
    for x, old in zip((K, V, W, pos), before):
        if old is not None and not in_place:
            assert torch.equal(x.view(torch.uint8), old.view(torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("T,keep,recent", [(1, 1, 0), (2, 1, 1), (5, 8, 3), (64, 64, 10), (65, 64, 0), (100, 1, 1), (1025, 1024, 256),
                                           (1000, 500, 500), (3001, 100, 50), (5000, 4999, 0), (20000, 2000, 64)])
def test_sizes(T, keep, recent, in_place):
    check(2, 3, T, 64, keep, recent, in_place=in_place, seed=T)


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kind", ["ties", "zeros", "mixed"])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("f32", 128)])
def test_ties_and_odd_weights(kind, dtype, d, in_place):
    check(2, 2, 1500, d, 300, 20, dtype, [1500, 1301], kind, True, in_place=in_place, kv_alloc=1510)
    check(3, 2, 700, d, 650, 0, dtype, [700, 640, 651], kind, False, False, in_place, seed=1)


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
def test_ragged_lengths(in_place):
    lens = [0, 1, 99, 100, 101, 300, -3, 999]
    check(8, 2, 300, 64, 100, 30, lens=lens, in_place=in_place, kv_alloc=305, out_alloc=120)
    check(8, 2, 300, 64, 100, 30, lens=lens, shuffled=True, in_place=in_place)
    check(8, 1, 300, 128, 100, 100, "f32", lens=lens, positions=False, in_place=in_place)


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(12))
def test_random(seed):
    rng = np.random.default_rng(9900 + seed)
    T = int(np.exp(rng.uniform(0, np.log(90000 if seed % 4 == 0 else 6000))))
    keep = int(rng.integers(1, T + 5))
    B = int(rng.integers(1, 4))
    check(B, int(rng.integers(1, 4)), T, int(rng.choice([64, 128])), keep, int(rng.integers(0, keep + 1)), str(rng.choice(["bf16", "f32"])),
          rng.integers(0, T + 1, B).tolist(), str(rng.choice(["floats", "ties", "mixed"])), bool(rng.random() < 0.5), bool(rng.random() < 0.7),
          bool(rng.random() < 0.5), T + int(rng.integers(0, 9)), seed=9900 + seed)


@pytest.mark.gpu
@pytest.mark.parametrize("T,keep", [(70000, 1000), (150000, 149000), (262144, 65536)])
def test_long_caches(T, keep):
    check(1, 2, T, 64, keep, 500, kind="ties", in_place=True, seed=T)
    check(1, 1, T, 64, keep, 0, seed=T)


@pytest.mark.gpu
def test_positions_at_the_ends_of_their_type():
    """newest - recent does not wrap around; equal positions are all recent, the lowest rows of them stay."""
    from paper_2603_15619_amd import moda_cache_evict

    K, V, W, _ = cache(1, 1, 40, 64, "bf16", 3)
    lo, hi = -(1 << 31), (1 << 31) - 1
    for fill, last in ((lo, lo + 2), (hi - 60, hi), (7, 7)):
        pos = torch.full((1, 1, 40), fill, dtype=torch.int32, device="cuda")
        pos[0, 0, -1] = last
        want, _ = R.evict_index(W.double().cpu().numpy(), 10, 5, pos.cpu().numpy())
        out = tuple(x[:, :, :10].clone().contiguous() for x in (K, V, W, pos))
        index, _ = moda_cache_evict(K, V, W, 10, 5, pos, out=out)
        assert np.array_equal(index.cpu().numpy(), want), fill


@pytest.mark.gpu
def test_step_by_step_in_place_and_captured():
    """A bounded cache: a row is written behind the kept ones, then one leaves, again and again, eager and from a graph."""
    from paper_2603_15619_amd import moda_cache_evict

    B, Hk, d, keep, recent = 2, 2, 64, 90, 30
    side = torch.cuda.Stream()
    for captured in (False, True):
        K, V, W, pos = cache(B, Hk, keep + 1, d, "bf16", 5)
        lengths = torch.tensor([keep, 40], dtype=torch.int32, device="cuda")
        new, index = torch.empty_like(lengths), torch.empty((B, Hk, keep), dtype=torch.int32, device="cuda")
        ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
        call = lambda: moda_cache_evict(K, V, W, keep, recent, pos, lengths, index=index, workspace=ws)
        if captured:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                call()
        for step in range(6):
            n = lengths.tolist()
            for b in range(B):  # the new token
                K[b, :, n[b]], V[b, :, n[b]] = torch.randn(Hk, d).cuda(), torch.randn(Hk, d).cuda()
                W[b, :, n[b]] = 0.0
                pos[b, :, n[b]] = 1000 + step
            W += torch.rand(W.shape).cuda()
            lengths += 1
            want, want_len = R.evict_index(W.double().cpu().numpy(), keep, recent, pos.cpu().numpy(), lengths.tolist())
            K0, pos0 = K.clone(), pos.clone()
            torch.cuda.synchronize()
            g.replay() if captured else call()
            torch.cuda.synchronize()
            assert np.array_equal(index.cpu().numpy(), want) and lengths.tolist() == want_len.tolist()
            at = torch.from_numpy(want).cuda().long().clamp(min=0)
            for b in range(B):
                m = want_len[b]
                assert torch.equal(pos[b, :, :m], pos0[b].gather(1, at[b, :, :m]))
                assert torch.equal(K[b, :, :m], K0[b].gather(1, at[b, :, :m, None].expand(Hk, m, d)))
                assert (pos[b, :, :m] == 1000 + step).any(-1).all()  # the newest is there


@pytest.mark.gpu
def test_binding_refusals():
    from paper_2603_15619_amd import MODAError, moda_cache_evict

    K, V, W, pos = cache(1, 1, 40, 64, "bf16", 3)
    for kw in (dict(keep=0), dict(keep=10, recent=11), dict(keep=10, recent=-1), dict(keep=10, T=41), dict(keep=10, T=0)):
        with pytest.raises(MODAError, match="shape"):
            moda_cache_evict(K, V, W, **kw)
    small = (K[:, :, :9].clone(), V[:, :, :9].clone(), W[:, :, :9].clone(), None)
    with pytest.raises(MODAError, match="shape"):
        moda_cache_evict(K, V, W, 10, out=small)
    with pytest.raises(MODAError, match="shape"):  # keys in place, values not
        moda_cache_evict(K, V, W, 10, out=(K, V.clone(), W, None))
    with pytest.raises(MODAError, match="NULL"):
        moda_cache_evict(K, V, W, 10, positions=pos, out=(K.clone(), V.clone(), W.clone(), None))
    with pytest.raises(ValueError, match="weights"):
        moda_cache_evict(K, V, W.double(), 10)


def test_refusals_without_gpu():
    from paper_2603_15619_amd.binding import MODAShape, lib

    ok = dict(B=2, Hq=2, Hk=2, T=16, d=128, depth_alloc=0, depth_count=0, causal=1, scale=0.0, dtype=1)
    names = ["K", "V", "w", "pos", "lens", "Ko", "Vo", "wo", "po", "lo", "index", "ws"]
    base = {n: 0x1000 * (i + 1) for i, n in enumerate(names)}

    def status(keep=8, recent=2, kv_alloc=16, out_alloc=8, ws_bytes=1 << 40, shape=None, **ptr):
        p = {n: ctypes.c_void_p(v) for n, v in dict(base, **ptr).items()}
        return lib().moda_cache_evict(*(p[n] for n in names[:11]), keep, recent, kv_alloc, out_alloc, p["ws"], ws_bytes,
                                      ctypes.byref(MODAShape(**dict(ok, **(shape or {})))), None)

    assert status(shape=dict(B=0)) == 0
    assert status(keep=0) == 2 and status(recent=9) == 2 and status(recent=-1) == 2 and status(kv_alloc=15) == 2
    assert status(out_alloc=7) == 2 and status(shape=dict(T=0)) == 2 and status(shape=dict(T=-1)) == 2
    assert status(shape=dict(d=100)) == 3 and status(shape=dict(dtype=3)) == 3
    for name in ("K", "V", "w", "Ko", "Vo", "wo", "index"):
        assert status(**{name: None}) == 1, name
    assert status(pos=None) == 1 and status(po=None) == 1
    for name in ("K", "V", "w", "pos", "Ko", "Vo", "wo", "po", "index", "ws"):
        assert status(**{name: 0x100008}) == 4, name
    assert status(lens=0x100002) == 4 and status(lo=0x100002) == 4
    place = dict(Ko=base["K"], Vo=base["V"], wo=base["w"], po=base["pos"])
    assert status(**place) == 2  # in place with another allocation
    for name in place:
        assert status(**{n: v for n, v in place.items() if n != name}, out_alloc=16) == 2, name
    assert status(ws=None) == 6 and status(ws_bytes=8) == 6
    need = lib().moda_cache_evict_workspace_bytes(8, ctypes.byref(MODAShape(**ok)))
    assert need > 0 and status(ws_bytes=need - 1) == 6
    assert status(shape=dict(B=1 << 22, Hq=256, Hk=256)) == 3  # more workgroups than a launch takes
    assert lib().moda_cache_evict(*([None] * 11), 1, 0, 1, 1, None, 0, None, None) == 1
