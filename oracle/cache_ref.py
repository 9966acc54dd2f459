"""fp64 numpy definitions of the operators on a shared and a bounded sequence cache (include/moda.h), for the tests.

Everything is spelled out per (sequence, head): the keys a query sees are concatenated, the softmax has two passes, an
eviction sorts.  Arrays are float64 (exact upcasts of what the kernels consume); lengths are lists or None."""
import numpy as np


def _filled(lengths, n, most):
    return [most] * n if lengths is None else [min(max(int(x), 0), most) for x in lengths]


def decode_step(Q, Kp, Vp, Ks, Vs, Kd=None, Vd=None, prefix_lengths=None, lengths=None, P=None, T=None, depth_count=None,
                scale=None):
    """{O [B,Hq,d], LSE [B,Hq], weights [B,Hk,kv_alloc], mag [B,Hq,d], logit [B,Hq]}: mag = sum of weight * |value|, logit =
    scale * the largest sum of |products| behind a logit (what the rounding of sums is proportional to)."""
    B, Hq, d = Q.shape
    Hk = (Kp if Ks is None else Ks).shape[1]
    G, scale = Hq // Hk, scale or d ** -0.5
    kv_alloc = 0 if Ks is None else Ks.shape[2]
    lens = _filled(lengths, B, kv_alloc if T is None else T)
    Np = 1 if Kp is None else Kp.shape[0]
    plens = _filled(prefix_lengths, Np, 0 if Kp is None else Kp.shape[2] if P is None else P)
    L = 0 if Kd is None else Kd.shape[2] if depth_count is None else depth_count
    r = {"O": np.zeros((B, Hq, d)), "LSE": np.full((B, Hq), -np.inf), "weights": np.zeros((B, Hk, kv_alloc)),
         "mag": np.zeros((B, Hq, d)), "logit": np.zeros((B, Hq))}
    for b in range(B):
        x, n = b // (B // Np), lens[b]
        for g in range(Hk):
            ks, vs = [np.zeros((0, d))], [np.zeros((0, d))]
            if n:
                ks, vs = ks + [Ks[b, g, :n]], vs + [Vs[b, g, :n]]
            if Kp is not None:
                ks, vs = ks + [Kp[x, g, :plens[x]]], vs + [Vp[x, g, :plens[x]]]
            if L:
                ks, vs = ks + [Kd[b, g, :L]], vs + [Vd[b, g, :L]]
            k, v = np.concatenate(ks), np.concatenate(vs)
            for h in range(g * G, g * G + G):
                s = scale * (k @ Q[b, h])
                m = s.max(initial=-np.inf)
                if m == -np.inf:
                    continue
                e = np.exp(s - m)
                r["LSE"][b, h] = m + np.log(e.sum())
                w = e / e.sum()
                r["O"][b, h], r["mag"][b, h] = w @ v, w @ np.abs(v)
                r["weights"][b, g, :n] += w[:n]
                r["logit"][b, h] = scale * (np.abs(k) @ np.abs(Q[b, h])).max()
    return r


def key_weights(Q, K, LSE, lengths=None, window=0, causal=True, scale=None):
    """weights [B, Hk, kv_alloc] of a prompt, and scale * the largest sum of |products| behind a logit, [B, Hk]."""
    B, Hq, T, d = Q.shape
    Hk = K.shape[1]
    G, scale = Hq // Hk, scale or d ** -0.5
    W, logit = np.zeros((B, Hk, K.shape[2])), np.zeros((B, Hk))
    for b, n in enumerate(_filled(lengths, B, T)):
        t = np.arange(max(0, n - window) if window else 0, n)
        for h in range(Hq):
            k = K[b, h // G, :n]
            with np.errstate(invalid="ignore"):
                w = np.exp(scale * (Q[b, h, t] @ k.T) - LSE[b, h, t][:, None])
            w[LSE[b, h, t] == -np.inf] = 0.0  # a query that sees nothing
            if causal:
                w[t[:, None] < np.arange(n)[None, :]] = 0.0
            W[b, h // G, :n] += w.sum(0)
            if len(t):
                logit[b, h // G] = max(logit[b, h // G], scale * (np.abs(Q[b, h, t]) @ np.abs(k).T).max())
    return W, logit


def evict_index(weights, keep, recent=0, positions=None, lengths=None, T=None):
    """index [B, Hk, min(keep, T)] and the new lengths."""
    B, Hk, kv_alloc = weights.shape
    T = kv_alloc if T is None else T
    n = min(keep, T)
    lens = _filled(lengths, B, T)
    index = np.full((B, Hk, n), -1, dtype=np.int32)
    for b in range(B):
        fit = min(lens[b], keep)
        for g in range(Hk):
            rows = np.arange(lens[b])
            w = weights[b, g, :lens[b]]
            p = rows if positions is None else positions[b, g, :lens[b]].astype(np.int64)
            recent_rows = p > p.max() - recent if lens[b] else p > 0
            # the last key counts first; recent rows are all alike; a NaN sorts behind everything, -0 beside 0
            best = np.lexsort((rows, np.where(recent_rows, 0.0, -w), ~recent_rows))[:fit]
            if len(best) < lens[b]:
                stay = set(best[best < fit].tolist())
                behind = iter(sorted(best[best >= fit].tolist()))
                index[b, g, :fit] = [r if r in stay else next(behind) for r in range(fit)]
            else:
                index[b, g, :fit] = rows
    return index, np.array([min(x, keep) for x in lens], dtype=np.int32)
