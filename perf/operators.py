"""The operators that serve a shared and a bounded sequence cache, as measurable cases.

  op "shared"   moda_attn_decode_shared   one new token per sequence; groups of sequences share a prefix
  op "weights"  moda_attn_decode_weights  one new token per sequence; every cached key's attention weight
                                          is added to its accumulator
  op "prompt"   moda_attn_weights         the accumulated attention weight of every key of a prompt
  op "evict"    moda_cache_evict          the cache shrinks to the recent and the heaviest rows

With B sequences, Hq query heads on Hk key/value heads, head dimension d, caches of T rows of which a
sequence's own length (`lengths_of`) is filled, L depth slots of La allocated ones, dtype "bf16" or "f32".
Where `own` is false a pass takes elementary torch operations in 32 bits, else the public entry points.
"""
import math

import numpy as np
import torch

own = False


def _case(op, B, Hq, Hk, T, d, name=None, **more):
    c = {"op": op, "B": B, "Hq": Hq, "Hk": Hk, "T": T, "d": d, "dtype": "bf16", "spread": 0.5}
    c.update(more)
    if name is not None:
        c["name"] = name
    return c


def _shared(B, Hq, Hk, T, d, L, P, Np=1, La=None, name=None, **more):
    return _case("shared", B, Hq, Hk, T, d, name, L=L, La=L if La is None else La, P=P, Np=Np, **more)


def _weights(B, Hq, Hk, T, d, L, La=None, name=None, **more):
    return _case("weights", B, Hq, Hk, T, d, name, L=L, La=L if La is None else La, **more)


def _prompt(B, Hq, Hk, T, d, window=0, causal=True, name=None, **more):
    return _case("prompt", B, Hq, Hk, T, d, name, window=window, causal=causal, **more)


def _evict(B, Hk, T, d, keep, recent, ordered=True, name=None, **more):
    return _case("evict", B, Hk, Hk, T, d, name, keep=keep, recent=recent, ordered=ordered, **more)


def listed():
    return [
        # four answers to one question in a short chat: the smallest shared call, where latency counts
        _shared(4, 16, 16, 40, 128, 15, 1003, La=16, name="shared_small"),
        # 32 sequences behind one long document, one head per key/value head
        _shared(32, 16, 16, 1000, 128, 15, 32768, name="shared_long_32k"),
        # 64 sequences behind one system prompt, eight query heads per key/value head: 512 queries read each key
        _shared(64, 64, 8, 500, 64, 64, 16384, name="shared_group_16k"),
        # eight prompts of ragged lengths with eight samples each
        _shared(64, 32, 8, 300, 128, 7, 2000, Np=8, La=16, name="shared_samples"),
        # one short chat whose cache is kept bounded
        _weights(1, 16, 16, 1003, 128, 15, La=16, name="weights_short"),
        # a batch of long ragged contexts, one head per key/value head
        _weights(8, 16, 16, 65536, 128, 15, name="weights_long_64k"),
        # the same with grouped queries and a middling context
        _weights(16, 64, 8, 4000, 64, 64, name="weights_group"),
        # the weights of a batch of whole prompts, as evictions by accumulated weight start from
        _prompt(8, 16, 16, 4096, 128, spread=0.0, name="prompt_layer_4k"),
        # a ragged batch of short prompts in full precision, judged by its last queries only
        _prompt(2, 16, 8, 1000, 128, window=64, dtype="f32", name="prompt_window_f32"),
        # one long prompt, eight heads per group
        _prompt(1, 64, 8, 16384, 64, name="prompt_group_16k"),
        # a batch of long prompts shrinks to 4096 rows before decoding starts
        _evict(8, 16, 32768, 128, 4096, 1024, name="evict_prompt_32k"),
        # one step of a small bounded cache in full precision, whose rows are out of order by now
        _evict(1, 8, 1090, 64, 1024, 256, ordered=False, dtype="f32", name="evict_step_f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: lengths over their logarithm, odd ones included; slots from none to 64; one to eight
    heads per group; batches cut to the work of the largest listed case."""
    op = rng.choice(["shared", "weights", "prompt", "evict"])
    d = rng.choice([64, 128])
    L = rng.choice([0, 1, 4, 7, 15, 31, 64])
    La = L + rng.choice([0, 0, 1, 5])
    G = rng.choice([1, 1, 2, 4, 5, 8])
    Hk = rng.choice([2, 4, 8, 16]) if G <= 2 else rng.choice([1, 2, 4, 8])
    spread = rng.choice([0.0, 0.3, 0.9])
    if op == "shared":
        P, T, Np = _log_int(rng, 50, 32768), _log_int(rng, 2, 2000), rng.choice([1, 1, 2, 5])
        Np = min(Np, max(1, (1 << 19) // (Hk * P)))
        per = min(_log_int(rng, 2, 64), max(1, (1 << 25) // (G * Hk * P * Np)), max(1, (1 << 18) // (Hk * T * Np)))
        return _shared(Np * per, G * Hk, Hk, T, d, L, P, Np, La, spread=spread)
    if op == "weights":
        T = _log_int(rng, 20, 65536)
        B = min(_log_int(rng, 1, 32), max(1, (1 << 22) // (Hk * T)))
        return _weights(B, G * Hk, Hk, T, d, L, La, spread=spread)
    if op == "prompt":
        f32 = rng.random() < 0.25
        T = _log_int(rng, 20, 2048 if f32 else 12000)
        window = rng.choice([0, 0, 1, 32, 100])
        B = min(_log_int(rng, 1, 8), max(1, (1 << (15 if f32 else 17)) // (G * Hk * T)))
        return _prompt(B, G * Hk, Hk, T, d, window, rng.random() < 0.85 or T > 6000, spread=spread,
                       dtype="f32" if f32 else "bf16")
    T = _log_int(rng, 30, 65536)
    keep = min(T, _log_int(rng, 8, T))
    B = min(_log_int(rng, 1, 16), max(1, (1 << 22) // (Hk * T)), max(1, (1 << 18) // (Hk * keep)))
    return _evict(B, Hk, T, d, keep, rng.choice([0, keep // 4, keep // 2]), rng.random() < 0.5, spread=spread,
                  dtype=rng.choice(["bf16", "bf16", "f32"]))


def _ragged(n, T, spread):
    """Lengths from T down to (1 - spread) T, the first one T."""
    return [T - int(T * spread) * (i * 7 % 16) // 15 for i in range(n)]


def lengths_of(case):
    return _ragged(case["B"], case["T"], case["spread"])


def prefix_lengths_of(case):
    return _ragged(case["Np"], case["P"], 0.5)


# ------------------------------------------------------------------------------------------ one pass
def prepare(case, seed):
    c = dict(case)
    B, Hq, Hk, T, d = (c[k] for k in ("B", "Hq", "Hk", "T", "d"))
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dt)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    st = {"case": c, "Kseq": normal(B, Hk, T, d), "lengths": ints(lengths_of(c))}
    if c["op"] in ("shared", "weights"):
        st["Q"], st["Vseq"] = normal(B, Hq, d), normal(B, Hk, T, d)
        st["Kdepth"], st["Vdepth"] = (normal(B, Hk, c["La"], d) if c["La"] else None for _ in range(2))
        # buffers that a serving loop keeps
        st["out"], st["lse"] = torch.empty_like(st["Q"]), torch.empty((B, Hq), dtype=torch.float32, device="cuda")
        st["workspace"] = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    if c["op"] == "shared":
        st["Kprefix"], st["Vprefix"] = normal(c["Np"], Hk, c["P"], d), normal(c["Np"], Hk, c["P"], d)
        st["prefix_lengths"] = ints(prefix_lengths_of(c))
    elif c["op"] == "weights":
        # what earlier steps have gathered, and where this step's sums go
        st["weights"] = torch.rand((B, Hk, T), generator=gen, device="cuda").square_()
        st["weights_out"] = torch.zeros_like(st["weights"])
    elif c["op"] == "prompt":
        st["Q"] = normal(B, Hq, T, d)
        st["LSE"] = _prompt_lse(st["Q"], st["Kseq"], c["causal"])  # as the forward pass of the layer leaves it
        st["weights_out"] = torch.zeros((B, Hk, T), device="cuda")
        st["workspace"] = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    elif c["op"] == "evict":
        st["Vseq"] = normal(B, Hk, T, d)
        # most keys gather little weight, a few much; equal ones among them
        u = torch.rand((B, Hk, T), generator=gen, device="cuda")
        st["weights"] = torch.where(u < 0.1, torch.zeros_like(u), (1.0 / (1.001 - u)).floor() if c["T"] < 2000 else 1.0 / (1.001 - u))
        pos = torch.arange(T, dtype=torch.int32, device="cuda").expand(B, Hk, T)
        if not c["ordered"]:  # a cache that has been shrunk before: newer rows in older rows' places
            n = st["lengths"][:, None, None]
            swapped = n - 1 - pos
            pos = 3 * torch.where((pos % 5 == 0) & (swapped % 5 == 0) & (swapped >= 0), swapped, pos)
        st["positions"] = pos.to(torch.int32).contiguous()
        n = min(c["keep"], T)
        st["out"] = (torch.zeros((B, Hk, n, d), dtype=dt, device="cuda"), torch.zeros((B, Hk, n, d), dtype=dt, device="cuda"),
                     torch.zeros((B, Hk, n), device="cuda"), torch.zeros((B, Hk, n), dtype=torch.int32, device="cuda"))
        st["lengths_out"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        st["index"] = torch.zeros((B, Hk, n), dtype=torch.int32, device="cuda")
        st["workspace"] = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")
    return st


def _prompt_lse(Q, K, causal):
    """Log-sum-exp of every query over the keys that it sees, [B, Hq, T] fp32."""
    B, Hq, T, d = Q.shape
    G, lse = Hq // K.shape[1], torch.empty((B, Hq, T), device=Q.device)
    for b in range(B):
        for g in range(K.shape[1]):
            kt = K[b, g].float().t().contiguous()
            for r0 in range(0, T, 2048):
                r1 = min(T, r0 + 2048)
                n = r1 if causal else T
                s = torch.matmul(Q[b, g * G:(g + 1) * G, r0:r1].float(), kt[:, :n].contiguous()) / math.sqrt(d)
                if causal:
                    rows, keys = torch.arange(r0, r1, device=Q.device), torch.arange(n, device=Q.device)
                    s.masked_fill_(keys[None, :] > rows[:, None], -math.inf)
                m = s.amax(-1)
                lse[b, g * G:(g + 1) * G, r0:r1] = m + torch.exp(s - m[..., None]).sum(-1).log()
    return lse


def run(state):
    op = state["case"]["op"]
    return (_own if own else _plain)[op](state)


def _own_shared(s):
    from paper_2603_15619_amd import moda_attn_decode_shared

    O, LSE = moda_attn_decode_shared(s["Q"], s["Kprefix"], s["Vprefix"], s["Kseq"], s["Vseq"], s["Kdepth"], s["Vdepth"],
                                     prefix_lengths=s["prefix_lengths"], lengths=s["lengths"], depth_count=s["case"]["L"],
                                     out=s["out"], lse=s["lse"], workspace=s["workspace"])
    return {"O": O, "LSE": LSE}


def _own_weights(s):
    from paper_2603_15619_amd import moda_attn_decode_weights

    O, LSE, W = moda_attn_decode_weights(s["Q"], s["Kseq"], s["Vseq"], s["weights"], s["Kdepth"], s["Vdepth"],
                                         lengths=s["lengths"], depth_count=s["case"]["L"], weights_out=s["weights_out"],
                                         out=s["out"], lse=s["lse"], workspace=s["workspace"])
    return {"O": O, "LSE": LSE, "weights": W}


def _own_prompt(s):
    from paper_2603_15619_amd import moda_attn_weights

    c = s["case"]
    return {"weights": moda_attn_weights(s["Q"], s["Kseq"], s["LSE"], window=c["window"], causal=c["causal"],
                                         lengths=s["lengths"], weights_out=s["weights_out"], workspace=s["workspace"])}


def _own_evict(s):
    from paper_2603_15619_amd import moda_cache_evict

    c = s["case"]
    index, lengths = moda_cache_evict(s["Kseq"], s["Vseq"], s["weights"], c["keep"], recent=c["recent"],
                                      positions=s["positions"], lengths=s["lengths"], out=s["out"],
                                      lengths_out=s["lengths_out"], index=s["index"], workspace=s["workspace"])
    K, V, W, P = s["out"]
    return {"K": K, "V": V, "weights": W, "positions": P, "index": index, "lengths": lengths}


# ------------------------------------------------------------------------------------------ the plain form
def _visible(n_rows, lengths):
    """[n, 1, 1, n_rows]: row j of sequence i is filled."""
    return (torch.arange(n_rows, device="cuda")[None, :] < lengths[:, None])[:, None, None, :]


def _plain_scores(q, k, visible=None):
    """q [n, Hk, m, d], k [n, Hk, rows, d]: fp32 logits [n, Hk, m, rows]."""
    s = torch.matmul(q, k.float().transpose(2, 3).contiguous()) / math.sqrt(q.shape[-1])
    return s if visible is None else s.masked_fill(~visible, -math.inf)


def _plain_step(s, with_prefix):
    """One softmax over the prefix (if any), the own rows and the slots: O, LSE and the own rows' weights."""
    c = s["case"]
    B, Hq, Hk, d, L = c["B"], c["Hq"], c["Hk"], c["d"], c["L"]
    G = Hq // Hk
    q = s["Q"].float().view(B, Hk, G, d)
    parts = [(_plain_scores(q, s["Kseq"], _visible(c["T"], s["lengths"])), s["Vseq"])]
    if L:
        parts.append((_plain_scores(q, s["Kdepth"][:, :, :L]), s["Vdepth"][:, :, :L]))
    if with_prefix:
        Np, n = c["Np"], B // c["Np"]
        qp = q.view(Np, n, Hk, G, d).transpose(1, 2).reshape(Np, Hk, n * G, d)
        sp = _plain_scores(qp, s["Kprefix"], _visible(c["P"], s["prefix_lengths"]))
        mp = sp.amax(-1).view(Np, Hk, n, G).transpose(1, 2).reshape(B, Hk, G)
    m = torch.stack([x.amax(-1) for x, _ in parts] + ([mp] if with_prefix else [])).amax(0)
    z, o = torch.zeros_like(m), torch.zeros_like(q)
    e = [torch.exp(x - m[..., None]) for x, _ in parts]
    for p, (_, v) in zip(e, parts):
        z += p.sum(-1)
        o += torch.matmul(p, v.float())
    if with_prefix:
        p = torch.exp(sp - m.view(Np, n, Hk, G).transpose(1, 2).reshape(Np, Hk, n * G, 1))
        z += p.sum(-1).view(Np, Hk, n, G).transpose(1, 2).reshape(B, Hk, G)
        o += torch.matmul(p, s["Vprefix"].float()).view(Np, Hk, n, G, d).transpose(1, 2).reshape(B, Hk, G, d)
    return ((o / z[..., None]).to(s["Q"].dtype).view(B, Hq, d), (m + z.log()).view(B, Hq), (e[0] / z[..., None]).sum(2))


def _plain_shared(s):
    O, LSE, _ = _plain_step(s, True)
    return {"O": O, "LSE": LSE}


def _plain_weights(s):
    O, LSE, w = _plain_step(s, False)
    filled = _visible(s["case"]["T"], s["lengths"])[:, 0]
    return {"O": O, "LSE": LSE, "weights": torch.where(filled, s["weights"] + w, torch.zeros_like(w))}


def _plain_prompt(s):
    c, Q, K = s["case"], s["Q"], s["Kseq"]
    B, Hq, Hk, T, d = (c[k] for k in ("B", "Hq", "Hk", "T", "d"))
    G, W = Hq // Hk, torch.zeros((B, Hk, T), device="cuda")
    lens = s["lengths"][:, None]
    t = torch.arange(T, device="cuda")
    counted = t[None, :] < lens
    filled = counted
    if c["window"]:
        counted = counted & (t[None, :] >= lens - c["window"])
    # a few batches of (sequence, group) at a time, a stretch of queries at a time
    for g in range(Hk):
        kt = K[:, g].float().transpose(1, 2).contiguous()
        for h in range(g * G, (g + 1) * G):
            for r0 in range(0, T, 2048):
                r1 = min(T, r0 + 2048)
                n = r1 if c["causal"] else T
                p = torch.exp(torch.matmul(Q[:, h, r0:r1].float(), kt[:, :, :n].contiguous()) / math.sqrt(d)
                              - s["LSE"][:, h, r0:r1, None])
                use = counted[:, r0:r1, None]
                if c["causal"]:
                    use = use & (t[None, None, :n] <= t[None, r0:r1, None])
                W[:, g, :n] += torch.where(use, p, torch.zeros_like(p)).sum(1)
    return {"weights": torch.where(filled[:, None], W, torch.zeros_like(W))}


def _plain_evict(s):
    c = s["case"]
    B, Hk, T, d, keep = c["B"], c["Hk"], c["T"], c["d"], c["keep"]
    W, pos, lens = s["weights"], s["positions"], s["lengths"][:, None, None]
    r = torch.arange(T, device="cuda").expand(B, Hk, T)
    filled = r < lens
    newest = torch.where(filled, pos, torch.full_like(pos, -1)).amax(-1, keepdim=True)
    # by class (recent, filled, empty), then by weight, then by row: two stable sorts, the last key first
    rank = torch.where(filled, 1 + (pos > newest - c["recent"]).int(), torch.zeros_like(pos))
    order = torch.sort(W, dim=-1, descending=True, stable=True).indices
    order = order.gather(-1, torch.sort(rank.gather(-1, order), dim=-1, descending=True, stable=True).indices)
    n = min(keep, T)
    lengths_out = s["lengths"].clamp(max=keep)
    fit = lengths_out[:, None, None]
    kept = torch.zeros((B, Hk, T), dtype=torch.bool, device="cuda")
    kept.scatter_(-1, order, (r < fit))
    # kept rows that lie behind the new length fill the holes below it, both in ascending order
    dest = torch.where(kept & (r < fit), r, torch.full_like(r, n))
    hole, mover = ~kept & (r < fit), kept & (r >= fit)
    holes = torch.sort(torch.where(hole, r, torch.full_like(r, T)), dim=-1).values
    nth = (mover.long().cumsum(-1) - 1).clamp(min=0)
    dest = torch.where(mover, holes.gather(-1, nth), dest)
    index = torch.full((B, Hk, n + 1), -1, dtype=torch.int64, device="cuda")
    index.scatter_(-1, dest.clamp(max=n), r)
    index = index[:, :, :n].contiguous()
    live = torch.arange(n, device="cuda")[None, None, :] < fit
    index = torch.where(live, index, torch.full_like(index, -1))
    at = index.clamp(min=0)

    def rows(x):
        y = x.gather(2, at[..., None].expand(B, Hk, n, d)) if x.dim() == 4 else x.gather(2, at)
        return torch.where(live[..., None] if x.dim() == 4 else live, y, torch.zeros_like(y))

    return {"K": rows(s["Kseq"]), "V": rows(s["Vseq"]), "weights": rows(W), "positions": rows(pos),
            "index": index.int(), "lengths": lengths_out}


_own = {"shared": _own_shared, "weights": _own_weights, "prompt": _own_prompt, "evict": _own_evict}
_plain = {"shared": _plain_shared, "weights": _plain_weights, "prompt": _plain_prompt, "evict": _plain_evict}


# ------------------------------------------------------------------------------------------ what it cannot do without
def work(case):
    """Bytes: every row that takes part read once, every output row written once.  Operations: 4 d per (query, key)
    pair of a decoding step (two products), 2 d per pair of a prompt (one product)."""
    c = case
    B, Hq, Hk, T, d = (c[k] for k in ("B", "Hq", "Hk", "T", "d"))
    e = 2 if c["dtype"] == "bf16" else 4
    lens = lengths_of(c)
    if c["op"] in ("shared", "weights"):
        rows, pairs = sum(lens) + B * c["L"], sum(lens) + B * c["L"]
        if c["op"] == "shared":
            pre = prefix_lengths_of(c)
            rows += sum(pre)
            pairs += sum(pre) * (B // c["Np"])
        moved = 8 * Hk * sum(lens) if c["op"] == "weights" else 0
        return {"bytes": 2 * e * d * Hk * rows + 2 * e * B * Hq * d + 4 * B * Hq + moved, "flops": 4 * d * Hq * pairs}
    if c["op"] == "prompt":
        rows = pairs = 0
        for n in lens:
            w = min(n, c["window"] or n)
            rows += w
            pairs += sum(range(n - w + 1, n + 1)) if c["causal"] else w * n
        return {"bytes": (e * d + 4) * Hq * rows + (e * d + 4) * Hk * sum(lens), "flops": 2 * d * Hq * pairs}
    kept = [min(n, c["keep"]) for n in lens]
    return {"bytes": Hk * (8 * sum(lens) + (4 * e * d + 8 + 4) * sum(kept)), "flops": 0}


# ------------------------------------------------------------------------------------------ the same in 64 bits
def _exact_evict(c, st, lens):
    """Every (sequence, head) on the host: the rows that stay, then who fills which hole."""
    B, Hk, T, d = c["B"], c["Hk"], c["T"], c["d"]
    n = min(c["keep"], T)
    W, pos = st["weights"].double().cpu().numpy(), st["positions"].cpu().numpy()
    index = np.full((B, Hk, n), -1, dtype=np.int32)
    for b in range(B):
        fit = min(lens[b], n)
        for g in range(Hk):
            w, p = W[b, g, :lens[b]], pos[b, g, :lens[b]]
            recent = p > p.max(initial=-1) - c["recent"]
            best = np.lexsort((np.arange(lens[b]), -w, ~recent))[:fit]
            stays = best[best < fit]
            index[b, g, stays] = stays
            index[b, g, np.setdiff1d(np.arange(fit), stays)] = np.sort(best[best >= fit])
    at = torch.from_numpy(index).cuda()
    out = {"index": at, "lengths": torch.tensor([min(x, n) for x in lens], dtype=torch.int32, device="cuda")}
    src = at.long().clamp(min=0)
    for name, x in (("K", st["Kseq"]), ("V", st["Vseq"]), ("weights", st["weights"]), ("positions", st["positions"])):
        out[name] = torch.zeros((B, Hk, n) + x.shape[3:], dtype=torch.int32 if name == "positions" else torch.float64, device="cuda")
        for b in range(B):
            for g in range(Hk):
                fit = min(lens[b], n)
                out[name][b, g, :fit] = x[b, g].index_select(0, src[b, g, :fit])
    return out


def exact(case, seed):
    c = case
    st = prepare(c, seed)
    B, Hq, Hk, T, d = (c[k] for k in ("B", "Hq", "Hk", "T", "d"))
    G, lens = Hq // Hk, lengths_of(c)
    if c["op"] == "evict":
        return _exact_evict(c, st, lens)
    f64 = dict(dtype=torch.float64, device="cuda")
    if c["op"] == "prompt":
        W = torch.zeros((B, Hk, T), **f64)
        for b, n in enumerate(lens):
            first = max(0, n - c["window"]) if c["window"] else 0
            for h in range(Hq):
                k = st["Kseq"][b, h // G, :n].double()
                for r0 in range(first, n, 2048):
                    r1 = min(n, r0 + 2048)
                    logits = k @ st["Q"][b, h, r0:r1].double().t().contiguous() * (d ** -0.5)
                    if c["causal"]:
                        logits += torch.full_like(logits, -math.inf).tril(-1 - r0)
                    W[b, h // G, :n] += torch.exp(logits - st["LSE"][b, h, r0:r1].double()).sum(1)
        return {"weights": W}
    O, LSE = torch.zeros((B, Hq, d), **f64), torch.zeros((B, Hq), **f64)
    W = torch.zeros((B, Hk, T), **f64)
    for b in range(B):
        for g in range(Hk):
            ks, vs = [st["Kseq"][b, g, :lens[b]]], [st["Vseq"][b, g, :lens[b]]]
            if c["L"]:
                ks.append(st["Kdepth"][b, g, :c["L"]])
                vs.append(st["Vdepth"][b, g, :c["L"]])
            if c["op"] == "shared":
                x = b // (B // c["Np"])
                n = prefix_lengths_of(c)[x]
                ks.append(st["Kprefix"][x, g, :n])
                vs.append(st["Vprefix"][x, g, :n])
            k, v = torch.cat(ks).double(), torch.cat(vs).double()
            logits = st["Q"][b, g * G:(g + 1) * G].double() @ k.t().contiguous() * (d ** -0.5)
            lse = torch.logsumexp(logits, 1)
            p = torch.exp(logits - lse[:, None])
            O[b, g * G:(g + 1) * G], LSE[b, g * G:(g + 1) * G] = p @ v, lse
            if c["op"] == "weights":
                W[b, g, :lens[b]] = st["weights"][b, g, :lens[b]].double() + p[:, :lens[b]].sum(0)
    return {"O": O, "LSE": LSE} if c["op"] == "shared" else {"O": O, "LSE": LSE, "weights": W}
