"""Refusals of the calls on a paged cache, all made on the host: nothing is launched."""
import ctypes

import pytest
import torch

NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = 1, 2, 3, 4, 6
S = dict(B=2, Hq=4, Hk=2, T=40, d=64, depth_alloc=3, depth_count=2, causal=1, scale=0.0, dtype=1)
X = dict(n_pages=9, page_rows=16, max_pages=3, type=1)
# pointer arguments of each call, those that may be NULL, those that hold 4-byte values
CALLS = {
    "append": (["K", "V", "table", "lengths", "counts", "Kpages", "Vpages", "Kscales", "Vscales", "Kbounds"], {"lengths", "counts", "Kbounds"}),
    "read": (["Kpages", "Vpages", "Kscales", "Vscales", "table", "lengths", "Kout", "Vout"], {"lengths"}),
    "select": (["Q", "Kbounds", "table", "lengths", "chosen"], {"lengths"}),
    "decode": (["Q", "Kpages", "Vpages", "Kscales", "Vscales", "table", "lengths", "selected", "Kdepth", "Vdepth", "O", "LSE"], {"lengths", "selected"}),
}
WORDS = {"table", "lengths", "counts", "chosen", "selected"}


def call(name, shape=None, pages=None, keep=4, first=1, recent=1, read_first=0, n_selected=2, ws=0x100000, ws_bytes=1, **ptrs):
    """The status of a call that is all right but for its workspace of one byte (select, decode), or (append, read) refused last for its
    first bounds or output, which is misaligned unless the caller gives it."""
    from paper_2603_15619_amd.binding import MODAPages, MODAShape, lib

    L, names = lib(), CALLS[name][0]
    at = {n: 0x1000 * (i + 1) for i, n in enumerate(names)}
    if name == "append":
        at["counts"] += 2
    if name == "read":
        at["lengths"] += 2
    at.update(ptrs)
    p = {n: ctypes.c_void_p(v) for n, v in at.items()}
    s = None if shape is False else ctypes.byref(MODAShape(**dict(S, **(shape or {}))))
    x = None if pages is False else ctypes.byref(MODAPages(**dict(X, **(pages or {}))))
    args = [p[n] for n in names]
    if name == "append":
        return L.moda_page_append(*args, x, s, None)
    if name == "read":
        return L.moda_page_read(*args, read_first, x, s, None)
    if name == "select":
        return L.moda_page_select(*args, keep, first, recent, ctypes.c_void_p(ws), ws_bytes, x, s, None)
    return L.moda_attn_decode_paged(*args[:8], n_selected, *args[8:], ctypes.c_void_p(ws), ws_bytes, x, s, None)


LAST = {"append": ALIGN, "read": ALIGN, "select": WORKSPACE, "decode": WORKSPACE}


@pytest.mark.parametrize("name", CALLS)
def test_pointers(name):
    assert call(name) == LAST[name]
    for n in CALLS[name][0]:
        got = call(name, **{n: 0})
        if n in CALLS[name][1]:  # (counts of append and lengths of read are what is misaligned here: without them the call would run)
            if (name, n) not in (("append", "counts"), ("read", "lengths")):
                assert got == LAST[name], n
        else:
            assert got == NULL, n
        if n in WORDS:
            assert call(name, **{n: 0x8002}) == ALIGN, n
            if LAST[name] != ALIGN:
                assert call(name, **{n: 0x8004}) == LAST[name], n
        else:
            assert call(name, **{n: 0x8008}) == ALIGN, n
    assert call(name, shape=False) == NULL and call(name, pages=False) == NULL
    for n in ("Kscales", "Vscales"):  # bf16 pages have none
        if n in CALLS[name][0]:
            assert call(name, pages=dict(type=0), **{n: 0}) == LAST[name]
    if name == "decode":
        assert call(name, Kdepth=0, shape=dict(depth_count=0)) == LAST[name]


@pytest.mark.parametrize("name", CALLS)
def test_pages_and_shape(name):
    for bad, status in ((dict(n_pages=0), SHAPE), (dict(n_pages=-1), SHAPE), (dict(max_pages=0), SHAPE), (dict(page_rows=0), SHAPE),
                        (dict(page_rows=8), UNSUPPORTED), (dict(page_rows=48), UNSUPPORTED), (dict(page_rows=512), UNSUPPORTED),
                        (dict(type=2), UNSUPPORTED), (dict(type=-1), UNSUPPORTED), (dict(max_pages=(1 << 26) + 1), UNSUPPORTED)):
        assert call(name, pages=bad) == status, bad
    for bad, status in ((dict(B=-1), SHAPE), (dict(Hk=0), SHAPE), (dict(d=96), UNSUPPORTED), (dict(dtype=0), UNSUPPORTED), (dict(dtype=7), UNSUPPORTED),
                        (dict(T=-1), SHAPE)):
        assert call(name, shape=bad) == status, bad
    used = {"append": (), "read": (), "select": ("Hq",), "decode": ("Hq", "depth_count", "scale", "depth_alloc")}[name]
    odd = {"Hq": (0, -3, 7), "depth_alloc": (-1, 1 << 20), "depth_count": (-2, 9), "causal": (2, -1), "scale": (float("nan"), float("inf"))}
    for field, values in odd.items():
        for v in values:
            got = call(name, shape={field: v})
            assert got in (SHAPE, UNSUPPORTED) if field in used else got == LAST[name], (field, v)
    assert call(name, shape=dict(B=0), **{n: 0 for n in CALLS[name][0]}) == 0  # nothing to do


def test_numbers_of_each_call():
    for name in ("select", "decode"):
        assert call(name, shape=dict(T=49)) == SHAPE and call(name, shape=dict(T=48)) == WORKSPACE  # three pages of 16 rows
        assert call(name, ws=0) == WORKSPACE and call(name, ws=0x8008, ws_bytes=1 << 40) == ALIGN
    for bad in (dict(keep=0), dict(keep=-1), dict(first=-1), dict(recent=-1), dict(keep=4, first=3, recent=2), dict(keep=4, first=1 << 30, recent=(1 << 31) - 1)):
        assert call("select", **bad) == SHAPE, bad
    assert call("read", read_first=-1) == SHAPE and call("read", read_first=(1 << 30) - 39) == UNSUPPORTED
    assert call("decode", n_selected=-1) == SHAPE and call("decode", n_selected=(1 << 26) + 1) == UNSUPPORTED
    assert call("append", shape=dict(T=0), K=0) == 0 and call("read", shape=dict(T=0), Kout=0) == 0
    # a grid of more than 2^32 threads
    big = dict(B=1 << 20, Hk=1 << 10, Hq=1 << 10)
    assert call("append", shape=big, counts=0) == UNSUPPORTED and call("read", shape=big, lengths=0) == UNSUPPORTED
    assert call("select", shape=big, ws_bytes=1 << 60) == UNSUPPORTED and call("decode", shape=big, ws_bytes=1 << 60) == UNSUPPORTED


def test_workspace_sizes():
    from paper_2603_15619_amd.binding import MODAPages, MODAShape, lib

    L, x = lib(), MODAPages(**X)
    size = lambda f, **s: f(ctypes.byref(x), ctypes.byref(MODAShape(**dict(S, **s))))
    assert size(L.moda_page_select_workspace_bytes, T=0) == 0 and size(L.moda_page_select_workspace_bytes, T=49) == 0
    assert size(L.moda_attn_decode_paged_workspace_bytes, B=0) == 0 and size(L.moda_attn_decode_paged_workspace_bytes, d=96) == 0
    need = [size(L.moda_page_select_workspace_bytes, T=t) for t in range(1, 49)]
    assert need == sorted(need) and need[0] > 0
    n = size(L.moda_attn_decode_paged_workspace_bytes)
    assert call("decode", ws_bytes=n - 1) == WORKSPACE and call("select", ws_bytes=need[39] - 1) == WORKSPACE


def cache(mx=False, n=6, Hk=2, R=16, d=64, B=2, device="cpu"):
    dt = torch.float8_e4m3fn if mx else torch.bfloat16
    r = dict(Kpages=torch.zeros(n, Hk, R, d, device=device).to(dt), Vpages=torch.zeros(n, Hk, R, d, device=device).to(dt),
             page_table=torch.zeros(B, 3, dtype=torch.int32, device=device))
    if mx:
        r.update(Kscales=torch.zeros(n, Hk, R, d // 32, dtype=torch.uint8, device=device), Vscales=torch.zeros(n, Hk, R, d // 32, dtype=torch.uint8, device=device))
    return r


def test_tensors_of_another_kind_are_refused():
    """(On host tensors, which are refused too: what is looked at before them, and that they are.)"""
    from paper_2603_15619_amd import moda_attn_decode_paged, moda_page_append, moda_page_read, moda_page_select

    Q, K = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 5, 64, dtype=torch.bfloat16)
    calls = (lambda **a: moda_page_append(K, K, **a), lambda **a: moda_page_read(**a), lambda **a: moda_attn_decode_paged(Q, **a))
    for f in calls:
        for a in (cache(), cache(True)):
            with pytest.raises(ValueError, match="device memory"):
                f(**a)
        with pytest.raises(TypeError, match="float8"):
            f(**dict(cache(), Kpages=torch.zeros(6, 2, 16, 64)))
        with pytest.raises(ValueError, match="scales"):
            f(**{k: v for k, v in cache(True).items() if k != "Vscales"})
        with pytest.raises(ValueError, match="scales"):
            f(**dict(cache(), Kscales=cache(True)["Kscales"]))
        with pytest.raises(ValueError, match="expected"):
            f(**dict(cache(), page_table=torch.zeros(2, dtype=torch.int32)))
        with pytest.raises(ValueError, match="expected"):
            f(**dict(cache(), Kpages=torch.zeros(6, 2, 64, dtype=torch.bfloat16)))
    for n in (1 << 31, (1 << 32) + 5, -(1 << 31) - 1):
        b = torch.zeros(6, 2, 2, 64, dtype=torch.bfloat16)
        for name in ("keep", "first", "recent", "T", "page_rows"):
            with pytest.raises(ValueError, match="%s: .*32 bits" % name):
                moda_page_select(Q, b, cache()["page_table"], **dict(dict(keep=2, page_rows=16), **{name: n}))


@pytest.mark.gpu
def test_shapes_types_and_strides_are_refused():
    from paper_2603_15619_amd import MODAError, moda_attn_decode_paged, moda_page_append, moda_page_read, moda_page_select

    c, m = cache(device="cuda"), cache(True, device="cuda")
    t = lambda *s, **k: torch.zeros(s, dtype=torch.bfloat16, device="cuda", **k)
    Q, K, lens = t(2, 4, 64), t(2, 2, 5, 64), torch.zeros(2, dtype=torch.int32, device="cuda")
    b = t(6, 2, 2, 64)
    for bad in (dict(Vpages=t(6, 2, 16, 128)), dict(Vpages=m["Vpages"]), dict(Kpages=t(2, 6, 16, 64).transpose(0, 1)), dict(page_table=c["page_table"].long()),
                dict(page_table=c["page_table"][:1]), dict(lengths=lens.long()), dict(lengths=lens[:1]), dict(page_table=torch.zeros(2, 6, dtype=torch.int32, device="cuda")[:, ::2])):
        for f in (lambda **a: moda_page_append(K, K, **a), lambda **a: moda_page_read(T=8, out=(t(2, 2, 8, 64), t(2, 2, 8, 64)), **a), lambda **a: moda_attn_decode_paged(Q, **a)):
            with pytest.raises(ValueError):
                f(**dict(c, **bad))
    for bad in (dict(Kscales=m["Kscales"][..., :1]), dict(Vscales=m["Vscales"].int())):
        with pytest.raises(ValueError):
            moda_page_read(**dict(m, **bad))
    for a, k in (((t(2, 3, 5, 64), K), {}), ((K, t(2, 2, 6, 64)), {}), ((K.float(), K.float()), {}), ((t(2, 2, 64, 5).transpose(2, 3), K), {}), ((K, K), dict(counts=lens[:1])),
                 ((K, K), dict(Kbounds=t(6, 2, 64))), ((K, K), dict(Kbounds=t(5, 2, 2, 64)))):
        with pytest.raises(ValueError):
            moda_page_append(*a, **c, **k)
    for k in (dict(Q=Q.float()), dict(Q=t(2, 4, 128)), dict(Q=t(3, 4, 64)), dict(Kdepth=t(2, 2, 3, 64), Vdepth=t(2, 2, 4, 64)), dict(selected=t(2, 2, 3).long()),
              dict(selected=torch.zeros(2, 2, 0, dtype=torch.int32, device="cuda")), dict(selected=torch.zeros(2, 4, dtype=torch.int32, device="cuda")),
              dict(out=t(2, 4, 32)), dict(lse=t(2, 4)), dict(workspace=torch.zeros(1 << 20))):
        with pytest.raises(ValueError):
            moda_attn_decode_paged(**dict(dict(c, Q=Q), **k))
    for k in (dict(Kbounds=b[:, :, 0]), dict(Kbounds=b.float()), dict(out=torch.zeros(2, 2, 3, dtype=torch.int32, device="cuda")), dict(lengths=lens.float())):
        with pytest.raises(ValueError):
            moda_page_select(**dict(dict(Q=Q, Kbounds=b, page_table=c["page_table"], keep=2, page_rows=16), **k))
    for f in (lambda: moda_attn_decode_paged(Q, **c, T=49), lambda: moda_page_select(Q, b, c["page_table"], 1, 16), lambda: moda_page_select(Q, b, c["page_table"], 2, 20),
              lambda: moda_attn_decode_paged(t(2, 3, 64), **c), lambda: moda_attn_decode_paged(Q, **c, workspace=t(8)), lambda: moda_page_read(**c, first=-1, T=4)):
        with pytest.raises(MODAError):
            f()
