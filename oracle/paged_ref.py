"""fp64 numpy definitions of the operators on a paged sequence cache (include/moda.h), for the tests.

Everything is spelled out row by row or page by page.  Arrays are float64 (exact upcasts of what the kernels consume); tables, lengths and
counts are integer arrays or lists, or None where the C ABI takes NULL."""
import numpy as np

# the 127 finite magnitudes of e4m3, in the order of their codes
E4M3 = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)])


def quantise(x):
    """[..., d] -> (values [..., d], exponents [..., d/32]): what 8-bit pages hold."""
    y = x.reshape(x.shape[:-1] + (-1, 32))
    finite = np.isfinite(y)
    a = np.where(finite, np.abs(y), 0.0).max(-1)
    e = np.full(a.shape, -100)
    while True:
        small = a > 448.0 * 2.0 ** e
        if not small.any():
            break
        e = np.where(small, e + 1, e)
    z = np.abs(y) / (2.0 ** e)[..., None]
    with np.errstate(invalid="ignore"):
        # (2^127 * 2 is no bf16 number: the largest magnitudes of all)
        z = np.where((e == 120)[..., None], np.minimum(z, 240.0), z)
        hi = np.clip(np.searchsorted(E4M3, np.where(finite, z, 0.0)), 0, 126)  # the first at or above
        lo = np.maximum(hi - 1, 0)
        up, down = E4M3[hi] - z, z - E4M3[lo]
        code = np.where((up < down) | ((up == down) & (hi % 2 == 0)) | (E4M3[hi] == z), hi, lo)
        v = np.sign(y) * E4M3[code] * (2.0 ** e)[..., None]
    return np.where(finite, v, np.nan).reshape(x.shape), e


def filled(lengths, b, most):
    return most if lengths is None else min(max(int(lengths[b]), 0), most)


def append(K, V, Kp, Vp, table, lengths=None, counts=None, mx=False, bounds=None):
    """In place on float64 pools [n_pages, Hk, R, d] (and bounds [n_pages, Hk, 2, d]); returns the written (page, row)s.  Row 0 of a page
    starts its bounds anew, every later row joins them."""
    B, Hk, T, d = K.shape
    n_pages, _, R, _ = Kp.shape
    written = []
    for b in range(B):
        length = T if lengths is None else max(int(lengths[b]), 0)
        n = min(T, length if counts is None else max(int(counts[b]), 0), length)
        for r in range(n):
            pos = length - n + r
            if pos // R >= table.shape[1] or not 0 <= table[b, pos // R] < n_pages:
                continue
            page, slot = int(table[b, pos // R]), pos % R
            for x, pool in ((K, Kp), (V, Vp)):
                pool[page, :, slot] = quantise(x[b, :, r])[0] if mx else x[b, :, r]
            written.append((page, slot))
            if bounds is not None:
                k = Kp[page, :, slot]
                if slot == 0:
                    bounds[page, :, 0] = bounds[page, :, 1] = k
                else:
                    bounds[page, :, 0] = np.minimum(bounds[page, :, 0], k)
                    bounds[page, :, 1] = np.maximum(bounds[page, :, 1], k)
                bad = np.isnan(bounds[page]).any(1)
                bounds[page][np.repeat(bad[:, None], 2, 1)] = np.nan
    return written


def read(Kp, Vp, table, K, V, lengths=None, first=0):
    """In place on K, V [B, Hk, T, d]."""
    B, _, T, _ = K.shape
    n_pages, _, R, _ = Kp.shape
    for b in range(B):
        for r in range(first, min(first + T, filled(lengths, b, table.shape[1] * R))):
            page = int(table[b, r // R])
            if 0 <= page < n_pages:
                K[b, :, r - first], V[b, :, r - first] = Kp[page, :, r % R], Vp[page, :, r % R]


def select(Q, bounds, table, keep, R, lengths=None, first=1, recent=1, T=None):
    """pages [B, Hk, keep]."""
    B, Hq, _ = Q.shape
    n_pages, Hk = bounds.shape[:2]
    G, T = Hq // Hk, table.shape[1] * R if T is None else T
    out = np.full((B, Hk, keep), -1, dtype=np.int32)
    for b in range(B):
        n = -(-filled(lengths, b, T) // R)
        pages = [p for p in range(n) if 0 <= table[b, p] < n_pages]
        for g in range(Hk):
            q = Q[b, g * G:g * G + G]
            scores = {}
            for p in pages:
                lo, hi = bounds[int(table[b, p]), g]
                with np.errstate(invalid="ignore"):  # (zero times an infinite bound is NaN, as the formula has it)
                    s = (np.maximum(q, 0).sum(0) * hi + np.minimum(q, 0).sum(0) * lo).sum()
                rank = 0 if p < first or p >= n - recent else 1
                order = 0.0 if rank == 0 else -s
                scores[p] = (rank, not np.isnan(order), 0.0 if np.isnan(order) else order, p)
            best = sorted(sorted(pages, key=lambda p: scores[p])[:keep])
            out[b, g, :len(best)] = best
    return out


def decode(Q, Kp, Vp, table, Kd=None, Vd=None, lengths=None, selected=None, T=None, depth_count=None, scale=None):
    """{O [B,Hq,d], LSE [B,Hq], mag [B,Hq,d], logit [B,Hq]} as cache_ref.decode_step gives them."""
    B, Hq, d = Q.shape
    n_pages, Hk, R, _ = Kp.shape
    G, scale = Hq // Hk, scale or d ** -0.5
    T = table.shape[1] * R if T is None else T
    L = 0 if Kd is None else Kd.shape[2] if depth_count is None else depth_count
    r = {"O": np.zeros((B, Hq, d)), "LSE": np.full((B, Hq), -np.inf), "mag": np.zeros((B, Hq, d)), "logit": np.zeros((B, Hq))}
    for b in range(B):
        n = filled(lengths, b, T)
        for g in range(Hk):
            listed = range(-(-n // R)) if selected is None else [int(p) for p in selected[b, g] if 0 <= p < -(-n // R)]
            ks, vs = [np.zeros((0, d))], [np.zeros((0, d))]
            for p in listed:
                page = int(table[b, p])
                if 0 <= page < n_pages:
                    ks.append(Kp[page, g, :min(R, n - p * R)])
                    vs.append(Vp[page, g, :min(R, n - p * R)])
            if L:
                ks, vs = ks + [Kd[b, g, :L]], vs + [Vd[b, g, :L]]
            k, v = np.concatenate(ks), np.concatenate(vs)
            for h in range(g * G, g * G + G):
                s = scale * (k @ Q[b, h])
                m = s.max(initial=-np.inf)
                if m == -np.inf:
                    continue
                e = np.exp(s - m)
                w = e / e.sum()
                r["LSE"][b, h] = m + np.log(e.sum())
                r["O"][b, h], r["mag"][b, h] = w @ v, w @ np.abs(v)
                r["logit"][b, h] = scale * (np.abs(k) @ np.abs(Q[b, h])).max()
    return r
