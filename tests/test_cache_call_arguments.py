"""Arguments of the calls on a shared or bounded cache that few callers pass: shape fields that a call does not use, numbers that
do not fit the C ABI's."""
import ctypes

import pytest

# fields of moda_shape, each with values that no call which uses it takes
ODD = {"Hq": (0, -3, 7), "depth_alloc": (-1, 1 << 20), "depth_count": (-2, 9), "causal": (2, -1), "scale": (float("nan"), float("inf"))}
USED_BY = {"evict": (), "weights": ("Hq", "causal", "scale"), "shared": ("Hq", "depth_alloc", "depth_count", "scale")}


def status(call, **odd):
    """The status of a call whose arguments are all right but for the last ones checked: a workspace of one byte, or (a call that
    takes none here) a misaligned output.  Nothing is launched."""
    from paper_2603_15619_amd.binding import MODAShape, lib

    # (two heads on two, so that Hq = 7 is no multiple)
    s = ctypes.byref(MODAShape(**dict(dict(B=2, Hq=2, Hk=2, T=16, d=64, depth_alloc=0, depth_count=0, causal=1, scale=0.0, dtype=1), **odd)))
    p = [ctypes.c_void_p(0x1000 * (i + 1)) for i in range(14)]
    L = lib()
    if call == "evict":
        return L.moda_cache_evict(*p[:11], 8, 2, 16, 8, p[11], 1, s, None)
    if call == "weights":
        return L.moda_attn_weights(*p[:5], ctypes.c_void_p(0x8008), 0, 16, None, 0, s, None)
    if call == "decode_weights":
        return L.moda_attn_decode_weights(*p[:10], 16, p[10], 1, s, None)
    return L.moda_attn_decode_shared(*p[:13], 16, p[13], 1, None, s, None)


@pytest.mark.parametrize("call,uses,last", [("evict", "evict", 6), ("weights", "weights", 4), ("shared", "shared", 6), ("decode_weights", "shared", 6)])
def test_fields_that_a_call_does_not_use_may_hold_anything(call, uses, last):
    assert status(call) == last
    for field, values in ODD.items():
        for v in values:
            got = status(call, **{field: v})
            if field in USED_BY[uses]:
                assert got in (2, 3), (field, v)
            else:
                assert got == last, (field, v)


def test_workspace_sizes_look_at_the_fields_in_use_only():
    from paper_2603_15619_amd.binding import MODAShape, lib

    base = dict(B=2, Hq=8, Hk=2, T=40000, d=64, depth_alloc=0, depth_count=0, causal=1, scale=0.0, dtype=1)
    L = lib()
    for uses, size in (("evict", lambda s: L.moda_cache_evict_workspace_bytes(100, s)), ("weights", lambda s: L.moda_attn_weights_workspace_bytes(0, s)),
                       ("shared", lambda s: L.moda_attn_decode_shared_workspace_bytes(None, 1, s))):
        # (a prompt of one tile of keys, so that the queries of its 64 heads are dealt out)
        b = dict(base, T=200, Hq=64, Hk=1, B=1) if uses == "weights" else base
        want = size(ctypes.byref(MODAShape(**b)))
        assert want > 0
        for field, values in ODD.items():
            if field not in USED_BY[uses]:
                for v in values:
                    assert size(ctypes.byref(MODAShape(**dict(b, **{field: v})))) == want, (uses, field, v)


def test_numbers_that_do_not_fit_32_bits_are_refused():
    """2^32 + 5 rows to keep are not 5.  (On the host: numbers are looked at before tensors.)"""
    import torch

    from paper_2603_15619_amd import moda_attn_decode_shared, moda_attn_decode_weights, moda_attn_weights, moda_cache_evict

    t, w = torch.zeros(2, 2, 8, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 8)
    q = t[:, :, 0].contiguous()
    calls = {"keep": lambda n: moda_cache_evict(t, t, w, n), "recent": lambda n: moda_cache_evict(t, t, w, 6, recent=n),
             "T": lambda n: moda_cache_evict(t, t, w, 6, T=n), "window": lambda n: moda_attn_weights(t, t, w, window=n, weights_out=w)}
    for n in (1 << 31, (1 << 32) + 5, -(1 << 32) + 5, -(1 << 31) - 1, 1 << 70):
        for name, call in calls.items():
            with pytest.raises(ValueError, match="%s: .*32 bits" % name):
                call(n)
        for name in ("P", "T", "depth_count"):
            with pytest.raises(ValueError, match="%s: .*32 bits" % name):
                moda_attn_decode_shared(q, t, t, t, t, t, t, **{name: n})
        for name in ("T", "depth_count"):
            with pytest.raises(ValueError, match="%s: .*32 bits" % name):
                moda_attn_decode_weights(q, t, t, w, t, t, **{name: n})
