"""The choice of pages in each of its forms, on both sides of the sizes where they change: one workgroup of 256 threads per (sequence, key/value head), one of
1024, or two kernels, whose first takes one batch of pages per wave or several.  Whole numbers, no tolerance; pages stand in several places of a table,
so that many scores are equal."""
import numpy as np
import pytest
import torch

from oracle import paged_ref as P
from paged_cases import f, ints, normal


def reference(Q, bounds, table, keep, R, lens, first, recent):
    """oracle.paged_ref.select, a sequence's pages at once."""
    B, Hq, _ = Q.shape
    n_pages, Hk = bounds.shape[:2]
    out = np.full((B, Hk, keep), -1, dtype=np.int32)
    for b in range(B):
        n = -(-max(0, min(int(lens[b]), table.shape[1] * R)) // R)
        pages = np.array([p for p in range(n) if 0 <= table[b, p] < n_pages], dtype=np.int64)
        if len(pages) == 0:
            continue
        q = Q[b].reshape(Hk, Hq // Hk, -1)
        up, down = np.maximum(q, 0).sum(1), np.minimum(q, 0).sum(1)
        x = bounds[table[b, pages]]
        score = (x[:, :, 1] * up + x[:, :, 0] * down).sum(-1)
        stays = (pages < first) | (pages >= n - recent)
        for g in range(Hk):
            s = score[:, g]
            best = np.sort(pages[np.lexsort((pages, -np.nan_to_num(s), ~np.isnan(s), ~stays))[:keep]])
            out[b, g, :len(best)] = best
    return out


def case(B, Hk, cols, d, seed, G=2, R=16, pool=1500):
    g = torch.Generator().manual_seed(seed)
    x = normal(g, 2, pool, Hk, d)
    bounds = torch.stack([torch.minimum(x[0], x[1]), torch.maximum(x[0], x[1])], 2).contiguous()
    bounds[7:8, :, 1, 3] = float("nan")
    bounds[8:11, :, 0, 5] = float("nan")
    table = torch.randint(0, pool, (B, cols), generator=g, dtype=torch.int32)
    table[torch.rand((B, cols), generator=g) < 0.1] = -1
    table[:, 5::97] = pool  # (no page either)
    lens = [int(n) for n in torch.randint(0, cols * R + 1, (B,), generator=g)]
    lens[0], lens[1], lens[2], lens[B - 1] = cols * R, 1, 0, cols * R - R + 1
    return normal(g, B, G * Hk, d), bounds, table, lens


def test_reference_is_the_oracle():
    for seed, keep, first, recent in ((0, 9, 1, 1), (1, 1, 0, 0), (2, 40, 3, 5), (3, 200, 1, 0)):
        Q, bounds, table, lens = case(4, 2, 90, 64, seed, pool=30)
        args = f(Q), f(bounds), table.numpy(), keep, 16, lens, first, recent
        assert np.array_equal(reference(*args), P.select(*args))


# (sequences, key/value heads, columns of the table): up to 64 (sequence, head)s (187 columns of d = 128 or 375 of d = 64 change the form), more (250 and
# 500, 4096), and more than 256 (1024, 4096)
SIZES = [(8, 8, 186), (8, 8, 188), (8, 8, 374), (8, 8, 376), (9, 8, 249), (9, 8, 251), (9, 8, 499), (9, 8, 501), (9, 8, 2100), (9, 8, 4096), (9, 8, 4097),
         (33, 8, 600), (33, 8, 1024), (33, 8, 1025), (33, 8, 4097)]


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,Hk,cols", SIZES)
def test_forms(B, Hk, cols, d):
    from paper_2603_15619_amd import moda_page_select

    Q, bounds, table, lens = case(B, Hk, cols, d, cols + B)
    args = Q.cuda(), bounds.cuda(), table.cuda()
    for keep, first, recent in ((cols // 4, 2, 3), (3, 1, 1), (cols, 0, 0), (5, 2, 3)):
        print("case", dict(B=B, Hk=Hk, cols=cols, d=d, keep=keep, first=first, recent=recent), flush=True)
        out = torch.full((B, Hk, keep), -9, dtype=torch.int32, device="cuda")
        moda_page_select(*args, keep, 16, lengths=ints(lens), first=first, recent=recent, out=out)
        torch.cuda.synchronize()
        assert np.array_equal(out.cpu().numpy(), reference(f(Q), f(bounds), table.numpy(), keep, 16, lens, first, recent))


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,Hk,cols", [(9, 8, 700), (9, 8, 4097), (33, 8, 700)])
def test_four_scores_only(B, Hk, cols, d):
    """So many equal scores that the choice ends among them, and rows all alike."""
    from paper_2603_15619_amd import moda_page_select

    Q, bounds, table, lens = case(B, Hk, cols, d, cols, pool=4)
    bounds = bounds.nan_to_num()
    bounds[3] = bounds[2]
    for keep in (1, 50, cols // 2):
        print("case", dict(B=B, Hk=Hk, cols=cols, d=d, keep=keep), flush=True)
        got = moda_page_select(Q.cuda(), bounds.cuda(), table.cuda(), keep, 16, lengths=ints(lens), first=0, recent=1)
        assert np.array_equal(got.cpu().numpy(), reference(f(Q), f(bounds), table.numpy(), keep, 16, lens, 0, 1))
