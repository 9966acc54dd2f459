"""The operators that serve a paged sequence cache, as measurable cases.

  op "append"  moda_page_append        new rows of every sequence go to their places in the pages, in 8 bits where
                                       the pages hold 8 bits (then moda_page_read gives back what they stand for)
  op "read"    moda_page_read          rows of the pages as one array again
  op "select"  moda_page_select        the pages whose key bounds promise the largest logits
  op "decode"  moda_attn_decode_paged  one new token per sequence over all its pages
  op "sparse"  moda_page_select, then moda_attn_decode_paged over the selected pages

With B sequences, Hq query heads on Hk key/value heads, head dimension d, pages of R rows in pools that all sequences
share, lengths from N down (`lengths_of`), L depth slots, `mx`: pages of 8-bit floats with a power-of-two scale per 32
channels, else of bf16.  `gone` pages of every sequence, the oldest but the first, have been given back.
Where `own` is false a pass takes elementary torch operations in 32 bits (scores of pages, which decide, in 64), else the
public entry points.
"""
import math

import numpy as np
import torch

own = False


def _case(op, B, Hq, Hk, N, d, R, mx=False, name=None, **more):
    c = {"op": op, "B": B, "Hq": Hq, "Hk": Hk, "N": N, "d": d, "R": R, "mx": mx, "spread": 0.5, "gone": 0, "L": 0, "T": 0, "keep": 0}
    c.update(more)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one step of a small batch: a row per sequence and head, the smallest call, where latency counts
        _case("append", 4, 8, 8, 1003, 128, 16, T=1, name="append_step_small"),
        # a batch of ragged prompts is written in 8 bits and read back for its own attention
        _case("append", 8, 8, 8, 4096, 128, 64, True, T=4096, name="append_prompt_mx"),
        # a chunk of ragged prompts goes behind what earlier chunks left, into small pages
        _case("append", 16, 16, 16, 1711, 64, 16, T=1003, name="append_chunk"),
        # the rows of a batch of long contexts become one array again
        _case("read", 4, 8, 8, 16384, 128, 16, T=16384, name="read_long"),
        # the last rows of ragged caches in 8 bits
        _case("read", 16, 16, 16, 2777, 64, 32, True, T=999, name="read_tail_mx"),
        # one short chat: the smallest attention call
        _case("decode", 1, 16, 16, 1003, 128, 16, L=15, spread=0.0, name="decode_small"),
        # long ragged contexts, one head per key/value head
        _case("decode", 8, 16, 16, 65536, 128, 64, L=15, name="decode_long_64k"),
        # a large ragged batch in 8 bits, eight query heads per key/value head
        _case("decode", 32, 64, 8, 16000, 128, 32, True, spread=0.9, name="decode_group_mx"),
        # many middling contexts, four heads per key/value head, pages given back behind a window
        _case("decode", 64, 32, 8, 2100, 64, 16, L=7, gone=20, name="decode_window"),
        # long contexts of which every key/value head reads the 48 pages that promise most
        _case("sparse", 16, 64, 8, 32768, 128, 64, keep=48, name="sparse_32k"),
        # the choice alone: a short chat with small pages
        _case("select", 1, 16, 8, 4000, 128, 16, keep=16, spread=0.0, name="select_small"),
        # ... and a batch of very long contexts
        _case("select", 32, 32, 8, 131072, 128, 64, keep=64, name="select_long_128k"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: lengths over their logarithm, odd ones included; every page size, 1 to 16 heads per group; batches cut
    to the work of the largest listed cases."""
    op = rng.choice(["append", "read", "decode", "decode", "sparse", "select"])
    d = rng.choice([64, 128])
    R = rng.choice([16, 32, 64, 128, 256])
    mx = rng.random() < 0.5
    G = rng.choice([1, 1, 2, 4, 5, 8, 16])
    Hk = rng.choice([2, 4, 8, 16]) if G <= 2 else rng.choice([1, 2, 4, 8])
    spread = rng.choice([0.0, 0.3, 0.9, 1.0])
    more = {"spread": spread}
    if op in ("append", "read"):
        N = _log_int(rng, 1, 20000)
        if op == "append" and rng.random() < 0.4:
            more["T"] = min(N, _log_int(rng, 1, 4))
            B = min(_log_int(rng, 1, 256), max(1, (1 << 18) // (Hk * N) if mx else (1 << 21) // (Hk * N)))
        else:
            more["T"] = rng.choice([N, min(N, _log_int(rng, 1, N))])
            B = min(_log_int(rng, 1, 64), max(1, (1 << 18) // (Hk * N)))
        return _case(op, B, Hk, Hk, N, d, R, mx, **more)
    more["gone"] = rng.choice([0, 0, 0, 5])
    if op == "decode":
        N = _log_int(rng, 1, 65536)
        B = min(_log_int(rng, 1, 128), max(1, (1 << 22) // (Hk * N)))
        return _case(op, B, G * Hk, Hk, N, d, R, mx, L=rng.choice([0, 1, 7, 15, 64]), **more)
    # (a choice that has something to choose: twice as many pages as are kept, some of them by their score)
    N = _log_int(rng, 16 * R, 65536 if op == "sparse" else 131072)
    more["keep"] = min(_log_int(rng, 3, 100), N // (2 * R))
    if op == "sparse":
        B = min(_log_int(rng, 1, 64), max(1, (1 << 22) // (Hk * N)))
        return _case(op, B, G * Hk, Hk, N, d, R, mx, L=rng.choice([0, 15]), **more)
    B = min(_log_int(rng, 1, 64), max(1, (1 << 22) * R // (8 * Hk * N)))
    return _case(op, B, G * Hk, Hk, N, d, R, mx, **more)


def _ragged(n, most, spread):
    """Numbers from `most` down to (1 - spread) most, the first one `most`."""
    return [most - int(most * spread) * (i * 7 % 16) // 15 for i in range(n)]


def lengths_of(case):
    return _ragged(case["B"], case["N"], case["spread"])


def counts_of(case):
    """New rows of every sequence (append)."""
    return [min(n, t) for n, t in zip(lengths_of(case), _ragged(case["B"], case["T"], 0.0 if case["T"] < 16 else case["spread"]))]


def first_of(case):
    """The first row that is read back: all T rows up to the longest length; what an append has written."""
    if case["op"] == "append":
        return min(n - t for n, t in zip(lengths_of(case), counts_of(case)))
    return case["N"] - case["T"]


def pages_of(case):
    """[B] lists of the logical pages that each sequence holds: those of its rows, less the ones given back."""
    R, gone = case["R"], case["gone"]
    return [[p for p in range(-(-n // R)) if not 1 <= p <= gone] for n in lengths_of(case)]


# ------------------------------------------------------------------------------------------ one pass
def prepare(case, seed):
    c = dict(case)
    op, B, Hq, Hk, N, d, R, mx = (c[k] for k in ("op", "B", "Hq", "Hk", "N", "d", "R", "mx"))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    # pages in the order in which a pool that has long been in use hands them out
    held = pages_of(c)
    n_pages = sum(len(x) for x in held) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").cpu()
    max_pages = -(-N // R) + 1
    table, at = torch.full((B, max_pages), -1, dtype=torch.int32), 0
    for b, x in enumerate(held):
        if x:
            table[b, torch.tensor(x)] = order[at:at + len(x)].int()
        at += len(x)
    st = {"case": c, "first": first_of(c), "table": table.cuda(), "lengths": ints(lengths_of(c)), "Kscales": None, "Vscales": None}
    if op != "select":  # (rows behind a length hold what earlier users of the page left)
        for x in ("K", "V"):
            pool = normal(n_pages, Hk, R, d)
            if mx:
                pool, st[x + "scales"] = _quantised(pool)
            st[x + "pages"] = pool
    if op in ("append", "read"):
        rows = N - st["first"]
        if op == "read" or mx:
            st["out"] = tuple(torch.zeros((B, Hk, rows, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if op == "append":
        st["K"], st["V"], st["counts"] = normal(B, Hk, c["T"], d), normal(B, Hk, c["T"], d), ints(counts_of(c))
        st["bounds"] = _bounds(st["Kpages"], st["Kscales"])
    if op in ("decode", "sparse"):
        st["Q"] = normal(B, Hq, d)
        st["Kdepth"], st["Vdepth"] = (normal(B, Hk, c["L"], d) if c["L"] else None for _ in range(2))
        # buffers that a serving loop keeps
        st["O"], st["LSE"] = torch.empty_like(st["Q"]), torch.empty((B, Hq), dtype=torch.float32, device="cuda")
    if op == "sparse":
        st["bounds"] = _bounds(st["Kpages"], st["Kscales"])
    elif op == "select":
        st["Q"] = normal(B, Hq, d)
        # bounds as pages of keys have them that lie together around something
        mid, half = normal(n_pages, Hk, d).mul_(0.5), normal(n_pages, Hk, d).mul_(0.3).add_(2.0).abs_()
        st["bounds"] = torch.stack([mid - half, mid + half], 2)
    if op in ("sparse", "select"):
        st["pages"] = torch.empty((B, Hk, c["keep"]), dtype=torch.int32, device="cuda")
    if op in ("decode", "sparse", "select"):
        st["workspace"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    return st


def run(state):
    op = state["case"]["op"]
    return (_own if own else _plain)[op](state)


def _own_append(s):
    from paper_2603_15619_amd import moda_page_append

    moda_page_append(s["K"], s["V"], s["Kpages"], s["Vpages"], s["table"], lengths=s["lengths"], counts=s["counts"],
                     Kscales=s["Kscales"], Vscales=s["Vscales"], Kbounds=s["bounds"])
    if not s["case"]["mx"]:
        return {"K": s["Kpages"], "V": s["Vpages"], "bounds": s["bounds"]}
    return dict(_own_read(s), bounds=s["bounds"])


def _own_read(s):
    from paper_2603_15619_amd import moda_page_read

    K, V = moda_page_read(s["Kpages"], s["Vpages"], s["table"], lengths=s["lengths"], first=s["first"],
                          Kscales=s["Kscales"], Vscales=s["Vscales"], out=s["out"])
    return {"K": K, "V": V}


def _own_select(s):
    from paper_2603_15619_amd import moda_page_select

    c = s["case"]
    return {"pages": moda_page_select(s["Q"], s["bounds"], s["table"], c["keep"], c["R"], lengths=s["lengths"], out=s["pages"],
                                      workspace=s["workspace"])}


def _own_decode(s, pages=None):
    from paper_2603_15619_amd import moda_attn_decode_paged

    O, LSE = moda_attn_decode_paged(s["Q"], s["Kpages"], s["Vpages"], s["table"], s["Kdepth"], s["Vdepth"],
                                    lengths=s["lengths"], selected=pages, Kscales=s["Kscales"], Vscales=s["Vscales"],
                                    out=s["O"], lse=s["LSE"], workspace=s["workspace"])
    return {"O": O, "LSE": LSE}


def _own_sparse(s):
    pages = _own_select(s)
    return dict(_own_decode(s, pages["pages"]), **pages)


# ------------------------------------------------------------------------------------------ the plain form
def _power(e):
    """2^e of whole numbers, exactly, fp32."""
    return ((e + 127) << 23).view(torch.float32)


def _quantised(x):
    """[..., d] -> e4m3 codes and scale bytes [..., d/32]: the least power of two, 2^-100 or more, that brings the largest of 32 values
    to 448 or below."""
    y = x.float().unflatten(-1, (-1, 32))
    a = y.abs().amax(-1)
    mantissa, exponent = torch.frexp(a)
    e = torch.where(mantissa <= 0.875, exponent - 9, exponent - 8).clamp(min=-100)
    e = torch.where(a == 0, torch.full_like(e, -100), e)
    return (y * _power(-e)[..., None]).to(torch.float8_e4m3fn).flatten(-2), (e + 127).to(torch.uint8)


def _values(codes, scales):
    if scales is None:
        return codes.float()
    return (codes.float().unflatten(-1, (-1, 32)) * _power(scales.int() - 127)[..., None]).flatten(-2)


def _bounds(pool, scales):
    x = _values(pool, scales)
    return torch.stack([x.amin(2), x.amax(2)], 2).to(torch.bfloat16)


def _take(x, index):
    """x[index], also of 8-bit floats."""
    return x.view(torch.uint8)[index].view(x.dtype) if x.dtype == torch.float8_e4m3fn else x[index]


def _rows(pool, scales, table, n=None):
    """Rows of the pages table [B, n] as fp32 [B, Hk, n R, d]; of missing pages those of page 0."""
    ids = table.clamp(min=0).long()
    x = _values(_take(pool, ids), None if scales is None else scales[ids])
    return x.transpose(1, 2).flatten(2, 3)


def _filled(s):
    """[B, max_pages R]: the rows that are there."""
    R = s["case"]["R"]
    r = torch.arange(s["table"].shape[1] * R, device="cuda")
    return (r[None, :] < s["lengths"][:, None]) & (s["table"] >= 0).repeat_interleave(R, 1)


def _plain_read(s):
    c, first = s["case"], s["first"]
    there = _filled(s)[:, None, first:c["N"], None]
    # (only the pages that hold such rows)
    lo, hi = first // c["R"], -(-c["N"] // c["R"])
    cut = slice(first - lo * c["R"], c["N"] - lo * c["R"])
    out = {}
    for x, to in zip("KV", s["out"]):
        rows = _rows(s[x + "pages"], s[x + "scales"], s["table"][:, lo:hi])[:, :, cut].to(torch.bfloat16)
        out[x] = torch.where(there, rows, to)
    return out


def _plain_append(s):
    c, R = s["case"], s["case"]["R"]
    n, t = s["lengths"][:, None], s["counts"][:, None]
    r = torch.arange(c["T"], device="cuda")[None, :]
    pos = n - t + r
    page = s["table"].gather(1, (pos // R).clamp(0, s["table"].shape[1] - 1).long())
    b, r = torch.where((r < t) & (page >= 0))
    page, pos = page[b, r].long(), pos[b, r]
    slot = (pos % R).long()
    stored = None
    for x in "KV":
        rows = s[x][b, :, r]
        if c["mx"]:
            codes, scales = _quantised(rows)
            s[x + "pages"].view(torch.uint8)[page, :, slot] = codes.view(torch.uint8)
            s[x + "scales"][page, :, slot] = scales
            rows = _values(codes, scales)
        else:
            s[x + "pages"][page, :, slot] = rows
        stored = rows.float() if stored is None else stored
    # bounds of the pages that rows went to: over these rows, and, unless the page's row 0 is among them, what was known
    new = torch.zeros(s["bounds"].shape[0], dtype=torch.bool, device="cuda")
    new[page[slot == 0]] = True
    old = s["bounds"].float()
    lo = torch.where(new[:, None, None], math.inf, old[:, :, 0]).index_reduce_(0, page, stored, "amin")
    hi = torch.where(new[:, None, None], -math.inf, old[:, :, 1]).index_reduce_(0, page, stored, "amax")
    s["bounds"][page] = torch.stack([lo, hi], 2).to(torch.bfloat16)[page]
    if c["mx"]:
        return dict(_plain_read(s), bounds=s["bounds"])
    return {"K": s["Kpages"], "V": s["Vpages"], "bounds": s["bounds"]}


def _plain_select(s):
    c = s["case"]
    Hk, keep, G = c["Hk"], c["keep"], c["Hq"] // c["Hk"]
    q = s["Q"].double().unflatten(1, (Hk, G))
    up, down = q.clamp(min=0).sum(2)[:, None], q.clamp(max=0).sum(2)[:, None]
    x = s["bounds"][s["table"].clamp(min=0).long()].double()  # [B, max_pages, Hk, 2, d]
    score = ((x[..., 1, :] * up).sum(-1) + (x[..., 0, :] * down).sum(-1)).transpose(1, 2).contiguous()
    n = ((s["lengths"] + c["R"] - 1) // c["R"])[:, None]
    p = torch.arange(s["table"].shape[1], device="cuda")[None, :]
    rank = torch.where((p < 1) | (p >= n - 1), 2, 1) * ((p < n) & (s["table"] >= 0))
    rank = rank[:, None].expand_as(score)
    # two stable sorts, the last key first
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices
    order = order.gather(-1, torch.sort(rank.gather(-1, order), dim=-1, descending=True, stable=True).indices)[..., :keep]
    far = torch.where(rank.gather(-1, order) > 0, order, torch.full_like(order, score.shape[-1])).sort(-1).values
    pages = torch.where(far < score.shape[-1], far, torch.full_like(far, -1)).int()
    return {"pages": torch.nn.functional.pad(pages, (0, keep - pages.shape[-1]), value=-1)}


def _plain_attention(s, K, V, there):
    """K, V [B, Hk, rows, d] fp32, there [B, Hk or 1, rows]: one softmax over these rows and the slots."""
    c = s["case"]
    B, Hq, Hk, d, L = (c[k] for k in ("B", "Hq", "Hk", "d", "L"))
    q = s["Q"].float().view(B, Hk, Hq // Hk, d)
    x = torch.matmul(q, K.transpose(2, 3).contiguous()) / math.sqrt(d)
    x = x.masked_fill(~there[:, :, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    if L:
        y = torch.matmul(q, s["Kdepth"].float().transpose(2, 3).contiguous()) / math.sqrt(d)
        m = torch.maximum(m, y.amax(-1, keepdim=True))
    ref = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = torch.exp(x - ref)
    z, o = e.sum(-1, keepdim=True), torch.matmul(e, V)
    if L:
        e = torch.exp(y - ref)
        z, o = z + e.sum(-1, keepdim=True), o + torch.matmul(e, s["Vdepth"].float())
    o = torch.where(z > 0, o / z, torch.zeros_like(o))
    return {"O": o.to(torch.bfloat16).view(B, Hq, d), "LSE": (ref + z.log()).view(B, Hq)}


def _plain_decode(s):
    K, V = (_rows(s[x + "pages"], s[x + "scales"], s["table"]) for x in "KV")
    return _plain_attention(s, K, V, _filled(s)[:, None])


def _plain_sparse(s):
    c, out = s["case"], _plain_select(s)
    B, Hk, R = c["B"], c["Hk"], c["R"]
    p = out["pages"].clamp(min=0).long()
    ids = s["table"].gather(1, p.flatten(1)).view_as(p).clamp(min=0).long()
    heads = torch.arange(Hk, device="cuda")[None, :, None]
    K, V = (_values(x, y).flatten(2, 3) for x, y in (
        (_take(s[n + "pages"], (ids, heads)), None if s[n + "scales"] is None else s[n + "scales"][ids, heads]) for n in "KV"))
    row = p[..., None] * R + torch.arange(R, device="cuda")
    there = (out["pages"] >= 0)[..., None] & (row < s["lengths"][:, None, None, None])
    return dict(_plain_attention(s, K, V, there.flatten(2)), **out)


_own = {"append": _own_append, "read": _own_read, "select": _own_select, "decode": _own_decode, "sparse": _own_sparse}
_plain = {"append": _plain_append, "read": _plain_read, "select": _plain_select, "decode": _plain_decode, "sparse": _plain_sparse}


# ------------------------------------------------------------------------------------------ what it cannot do without
def _held_rows(case, pages):
    """Rows of one sequence's pages, of length n each."""
    return sum(min(case["R"], n - p * case["R"]) for n, x in zip(lengths_of(case), pages) for p in x)


def work(case):
    """Bytes: every row and bound that takes part read once, every output written once.  Operations: 4 d per (row, query head) of
    attention, 4 d per (page, key/value head) of a choice."""
    c = case
    op, B, Hq, Hk, d, R = (c[k] for k in ("op", "B", "Hq", "Hk", "d", "R"))
    stored = d + d // 32 if c["mx"] else 2 * d  # a row of K or V
    lens = lengths_of(c)
    bytes_ = flops = 0
    if op == "append":
        counts = counts_of(c)
        bytes_ += 2 * Hk * sum(counts) * (2 * d + stored)
        bytes_ += 4 * d * Hk * sum(-(-n // R) - (n - t) // R for n, t in zip(lens, counts) if t)
    if op == "read" or op == "append" and c["mx"]:
        bytes_ += 2 * Hk * sum(max(0, n - first_of(c)) for n in lens) * (2 * d + stored)
    held = pages_of(c)
    if op in ("select", "sparse"):
        bytes_ += 4 * d * Hk * sum(len(x) for x in held) + 2 * B * Hq * d + 4 * B * Hk * c["keep"]
        flops += 4 * d * Hk * sum(len(x) for x in held)
        held = [x if len(x) <= c["keep"] else x[len(x) - c["keep"]:] for x in held]  # (as many pages, the last one, not full, among them)
    if op in ("decode", "sparse"):
        rows = _held_rows(c, held)
        bytes_ += 2 * Hk * (rows * stored + B * c["L"] * 2 * d) + 4 * B * Hq * d + 4 * B * Hq
        flops += 4 * d * Hq * (rows + B * c["L"])
    return {"bytes": bytes_, "flops": flops}


# ------------------------------------------------------------------------------------------ the same in 64 bits
def _exact_stored(x, mx):
    """[..., d] bf16 -> what the pages then hold, in 64 bits: 8 values per octave, steps of 2^-9 below 2^-6, in units of the scale."""
    y = x.double()
    if not mx:
        return y
    shape = y.shape
    y = y.reshape(*shape[:-1], -1, 32)
    a = y.abs().amax(-1, keepdim=True)
    # the least power of two that will do, from one that will not
    e = torch.floor(torch.log2(torch.where(a > 0, a, torch.full_like(a, 2.0 ** -100)) / 448.0)) - 1.0
    for _ in range(3):
        e = torch.where(a <= 448.0 * torch.pow(2.0, e), e, e + 1.0)
    e = e.clamp(min=-100.0)
    unit = torch.pow(torch.full_like(e, 2.0), e)
    z = (y / unit).abs()
    step = torch.full_like(z, 2.0 ** -9)
    for k in range(-5, 9):
        step = torch.where(z >= 2.0 ** k, 2.0 ** (k - 3), step)
    return (torch.round(z / step) * step * torch.sign(y) * unit).reshape(shape)


def _exact_pool(s, x):
    """The pool in 64 bits, from codes and bytes where it is in 8 bits."""
    if s[x + "scales"] is None:
        return s[x + "pages"].double()
    unit = torch.pow(torch.tensor(2.0, dtype=torch.float64, device="cuda"), s[x + "scales"].double() - 127)
    return s[x + "pages"].double() * unit.repeat_interleave(32, dim=-1)


def _exact_append(c, s):
    R, table = c["R"], s["table"].cpu().numpy()
    lens, counts, first = lengths_of(c), counts_of(c), s["first"]
    pools = {x: _exact_pool(s, x) for x in "KV"}
    bounds = s["bounds"].double()
    for b, (n, t) in enumerate(zip(lens, counts)):
        new = {x: _exact_stored(s[x][b, :, :t], c["mx"]) for x in "KV"}
        for p in range((n - t) // R, -(-n // R) if t else 0):
            lo, hi = max(p * R, n - t), min(p * R + R, n)
            at = int(table[b, p])
            for x in "KV":
                pools[x][at, :, lo - p * R:hi - p * R] = new[x][:, lo - n + t:hi - n + t]
            rows = new["K"][:, lo - n + t:hi - n + t]
            if lo > p * R:
                rows = torch.cat([rows, bounds[at]], 1)
            bounds[at] = torch.stack([rows.min(1).values, rows.max(1).values], 1)
    if c["mx"]:
        return dict(_exact_read(c, s, pools, first), bounds=bounds)
    return dict(pools, bounds=bounds)


def _exact_read(c, s, pools, first):
    R, table, out = c["R"], s["table"].cpu().numpy(), {}
    for x in "KV":
        out[x] = torch.zeros(s["out"][0].shape, dtype=torch.float64, device="cuda")
        for b, n in enumerate(lengths_of(c)):
            for p in range(first // R, -(-n // R)):
                lo, hi = max(first, p * R), min(n, p * R + R)
                if lo < hi and table[b, p] >= 0:
                    out[x][b, :, lo - first:hi - first] = pools[x][int(table[b, p]), :, lo - p * R:hi - p * R]
    return out


def _exact_select(c, s):
    """Every (sequence, head) on the host."""
    B, Hk, G, keep = c["B"], c["Hk"], c["Hq"] // c["Hk"], c["keep"]
    Q, table = s["Q"].double().cpu().numpy(), s["table"].cpu().numpy()
    bounds = s["bounds"].float().cpu().numpy()
    pages = np.full((B, Hk, keep), -1, dtype=np.int32)
    for b, n in enumerate(lengths_of(c)):
        count = -(-n // c["R"])
        p = np.array([i for i in range(count) if table[b, i] >= 0], dtype=np.int64)
        for g in range(Hk):
            q = Q[b, g * G:g * G + G]
            x = bounds[table[b, p], g].astype(np.float64)
            score = x[:, 1] @ np.where(q > 0, q, 0).sum(0) + x[:, 0] @ np.where(q < 0, q, 0).sum(0)
            forced = (p == 0) | (p == count - 1)
            best = np.sort(p[np.lexsort((p, -score, ~forced))[:keep]])
            pages[b, g, :len(best)] = best
    return {"pages": torch.from_numpy(pages).cuda()}


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    op, B, Hq, Hk, d, R, L = (c[k] for k in ("op", "B", "Hq", "Hk", "d", "R", "L"))
    if op == "append":
        return _exact_append(c, s)
    if op == "read":
        return _exact_read(c, s, {x: _exact_pool(s, x) for x in "KV"}, s["first"])
    chosen = _exact_select(c, s) if op in ("select", "sparse") else {}
    if op == "select":
        return chosen
    f64 = dict(dtype=torch.float64, device="cuda")
    O, LSE = torch.zeros((B, Hq, d), **f64), torch.full((B, Hq), -math.inf, **f64)
    G, held, table = Hq // Hk, pages_of(c), s["table"].cpu()
    lists = chosen["pages"].cpu() if chosen else None
    for b, n in enumerate(lengths_of(c)):
        for g in range(Hk):
            mine = [p for p in lists[b, g].tolist() if p >= 0] if chosen else held[b]
            parts = {"K": [], "V": []}
            for x in "KV":
                if mine:
                    ids = table[b, torch.tensor(mine)].long().cuda()
                    rows = _take(s[x + "pages"][:, g], ids)
                    if c["mx"]:
                        unit = torch.pow(torch.tensor(2.0, **f64), s[x + "scales"][ids, g].double() - 127)
                        rows = rows.double() * unit.repeat_interleave(32, dim=-1)
                    rows = rows.double().reshape(-1, d)
                    at = (torch.tensor(mine, device="cuda")[:, None] * R + torch.arange(R, device="cuda")).reshape(-1)
                    parts[x].append(rows[at < n])
                if L:
                    parts[x].append(s[x + "depth"][b, g].double())
            if not parts["K"]:
                continue
            k, v = torch.cat(parts["K"]), torch.cat(parts["V"])
            logits = s["Q"][b, g * G:g * G + G].double() @ k.t().contiguous() * (d ** -0.5)
            lse = torch.logsumexp(logits, 1)
            O[b, g * G:g * G + G], LSE[b, g * G:g * G + G] = torch.exp(logits - lse[:, None]) @ v, lse
    return dict({"O": O, "LSE": LSE}, **chosen)
