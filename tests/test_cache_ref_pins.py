"""What pins the fp64 definitions of oracle/cache_ref.py: the oracle of the plain operator, library softmax, closed forms and a
literal sort."""
import numpy as np
import pytest
import torch

from oracle import cache_ref as C
from oracle import moda_ref as R


def arrays(seed, *shapes):
    rng = np.random.default_rng(seed)
    return [rng.standard_normal(s) for s in shapes]


def test_a_step_without_prefix_is_the_last_row_of_the_forward():
    Q, K, V, Kd, Vd = arrays(1, (2, 6, 16), (2, 2, 30, 16), (2, 2, 30, 16), (2, 2, 4, 16), (2, 2, 4, 16))
    r = C.decode_step(Q, None, None, K, V, Kd, Vd)
    O, L = R.fwd_rows(Q[:, :, None], K, V, Kd[:, :, None], Vd[:, :, None], np.array([29], dtype=np.int32))
    assert np.abs(r["O"] - O[:, :, 0]).max() <= 1e-12 and np.abs(r["LSE"] - L[:, :, 0]).max() <= 1e-12


def test_a_prefix_is_rows_that_every_sequence_holds():
    Q, K, V, Kp, Vp = arrays(2, (6, 4, 8), (6, 2, 9, 8), (6, 2, 9, 8), (3, 2, 11, 8), (3, 2, 11, 8))
    plens, lens = [11, 0, 5], [9, 0, 3, 1, 9, 2]
    r = C.decode_step(Q, Kp, Vp, K, V, prefix_lengths=plens, lengths=lens)
    for b in range(6):
        k, v = (np.concatenate([p[b // 2, :, :plens[b // 2]], x[b, :, :lens[b]]], 1)[None] for p, x in ((Kp, K), (Vp, V)))
        one = C.decode_step(Q[b:b + 1], None, None, k, v)
        assert np.abs(one["O"] - r["O"][b]).max() <= 1e-12 and np.abs(one["LSE"] - r["LSE"][b]).max() <= 1e-12
        n = plens[b // 2]
        assert np.abs(one["weights"][0, :, n:] - r["weights"][b, :, :lens[b]]).max(initial=0) <= 1e-12
        assert np.abs(one["weights"].sum(-1) - 2).max() <= 1e-12  # two heads per group


def test_nothing_seen():
    Q, K, V = arrays(3, (2, 2, 8), (2, 1, 5, 8), (2, 1, 5, 8))
    r = C.decode_step(Q, None, None, K, V, lengths=[0, -2])
    assert not r["O"].any() and np.all(r["LSE"] == -np.inf) and not r["weights"].any()


@pytest.mark.parametrize("causal", [True, False])
def test_key_weights_are_the_column_sums_of_the_softmax(causal):
    Q, K = arrays(4, (2, 4, 13, 8), (2, 2, 13, 8))
    s = torch.from_numpy(Q) @ torch.from_numpy(np.repeat(K, 2, 1)).transpose(2, 3) * 8 ** -0.5
    if causal:
        s = s.masked_fill(torch.ones(13, 13, dtype=torch.bool).triu(1), float("-inf"))
    p = torch.softmax(s, -1).view(2, 2, 2, 13, 13).sum(2).numpy()
    lse = torch.logsumexp(s, -1).numpy()
    W, _ = C.key_weights(Q, K, lse, causal=causal)
    assert np.abs(W - p.sum(2)).max() <= 1e-12
    W, _ = C.key_weights(Q, K, lse, window=4, causal=causal)
    assert np.abs(W - p[:, :, 9:].sum(2)).max() <= 1e-12
    W, _ = C.key_weights(Q, K, lse, lengths=[7, 0], window=3, causal=causal)
    assert np.abs(W[0, :, :7] - p[0, :, 4:7, :7].sum(1)).max() <= 1e-12 and not W[0, :, 7:].any() and not W[1].any()


def test_eviction_by_a_literal_reading_of_its_order():
    rng = np.random.default_rng(5)
    for _ in range(200):
        T, keep = int(rng.integers(1, 20)), int(rng.integers(1, 22))
        recent = int(rng.integers(0, keep + 1))
        w = np.floor(rng.random(T) * 4)
        w[rng.random(T) < 0.1] = np.nan
        pos = rng.permutation(T) * 2
        n = int(rng.integers(0, T + 1))
        newest = max(pos[:n], default=0)
        rank = sorted(range(n), key=lambda r: ((0, 0) if pos[r] > newest - recent else (1, np.inf if np.isnan(w[r]) else -w[r]), r))
        stay = set(rank[:keep])
        fit = min(n, keep)
        holes, movers = [r for r in range(fit) if r not in stay], sorted(r for r in stay if r >= fit)
        want = list(range(fit)) + [-1] * (min(keep, T) - fit)
        for hole, mover in zip(holes, movers):
            want[hole] = mover
        got, new = C.evict_index(w[None, None], keep, recent, pos[None, None], [n], T)
        assert got[0, 0].tolist() == want and new.tolist() == [fit]
