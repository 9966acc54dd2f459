"""Binding of the libmoda C ABI (include/moda.h).

Argument marshalling only: torch tensors supply device memory and the stream;
every step of the attention runs in the HIP kernels of libmoda.so.  There is no
fallback: if the library is missing or a call is rejected, an exception is raised.

Plain valid calls of moda_attn_fwd, moda_attn_bwd, moda_attn_decode, moda_depth_append and of the calls on a shared,
bounded or paged cache are marshalled by moda_torch.so (bind_csrc/moda_torch.cpp); whatever it declines comes back as None and is taken here,
through ctypes, with the same checks and an exception for the one that fails.
"""
import ctypes
import importlib.machinery
import importlib.util
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
# MODA_LIB_PATH points at another build of the same library (e.g. an experiment)
LIB_PATH = os.environ.get("MODA_LIB_PATH") or os.path.join(HERE, "libmoda.so")
NATIVE_PATH = os.path.join(HERE, "moda_torch.so")

MODA_F32, MODA_BF16 = 0, 1
MODA_PAGES_BF16, MODA_PAGES_MX8 = 0, 1
EXPORTS = ("moda_attn_fwd", "moda_attn_fwd_tuned", "moda_attn_bwd_workspace_bytes", "moda_attn_bwd", "moda_depth_append",
           "moda_attn_decode", "moda_attn_decode_workspace_bytes", "moda_attn_decode_noalloc",
           "moda_attn_decode_noalloc_max_bytes",
           "moda_attn_decode_shared", "moda_attn_decode_shared_workspace_bytes", "moda_attn_decode_weights",
           "moda_attn_weights", "moda_attn_weights_workspace_bytes",
           "moda_cache_evict", "moda_cache_evict_workspace_bytes",
           "moda_page_append", "moda_page_read", "moda_page_select", "moda_page_select_workspace_bytes",
           "moda_attn_decode_paged", "moda_attn_decode_paged_workspace_bytes",
           "moda_calibrate_mfma", "moda_calibrate_mfma_operand_bytes", "moda_calibrate_mfma_sink_bytes",
           "moda_status_string", "moda_version", "moda_kernels_per_call", "moda_fwd_kernel_name",
           "moda_bwd_kernel_name")


class MODAShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hk", ctypes.c_int32),
                ("T", ctypes.c_int32), ("d", ctypes.c_int32), ("depth_alloc", ctypes.c_int32),
                ("depth_count", ctypes.c_int32), ("causal", ctypes.c_int32),
                ("scale", ctypes.c_float), ("dtype", ctypes.c_int32)]


class MODAFwdTuning(ctypes.Structure):
    _fields_ = [("waves", ctypes.c_int32), ("heads_per_tile", ctypes.c_int32), ("head_group", ctypes.c_int32),
                ("depth_path", ctypes.c_int32)]


class MODAPrefix(ctypes.Structure):
    _fields_ = [("n_prefixes", ctypes.c_int32), ("prefix_rows", ctypes.c_int32), ("prefix_alloc", ctypes.c_int32)]


class MODAPages(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int32), ("page_rows", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("type", ctypes.c_int32)]


class MODAError(RuntimeError):
    def __init__(self, code, text):
        super().__init__("libmoda: %s (status %d)" % (text, code))
        self.code = code


_lib = None


def lib():
    """Load libmoda.so (built by paper_2603_15619_amd.build).  Raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                "%s not found: build it with `python -m paper_2603_15619_amd.build`" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        vp = ctypes.c_void_p
        sp = ctypes.POINTER(MODAShape)
        L.moda_attn_fwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, sp, vp]
        L.moda_attn_fwd.restype = ctypes.c_int
        L.moda_attn_fwd_tuned.argtypes = [vp, vp, vp, vp, vp, vp, vp, sp, ctypes.POINTER(MODAFwdTuning), vp]
        L.moda_attn_fwd_tuned.restype = ctypes.c_int
        L.moda_attn_bwd_workspace_bytes.argtypes = [sp]
        L.moda_attn_bwd_workspace_bytes.restype = ctypes.c_size_t
        L.moda_attn_bwd.argtypes = [vp] * 14 + [ctypes.c_size_t, sp, vp]
        L.moda_attn_bwd.restype = ctypes.c_int
        L.moda_depth_append.argtypes = [vp, vp, vp, vp, ctypes.c_int32, sp, vp]
        L.moda_depth_append.restype = ctypes.c_int
        L.moda_attn_decode_workspace_bytes.argtypes = [sp]
        L.moda_attn_decode_workspace_bytes.restype = ctypes.c_size_t
        L.moda_attn_decode.argtypes = [vp] * 7 + [ctypes.c_int32, vp, ctypes.c_size_t, sp, vp]
        L.moda_attn_decode.restype = ctypes.c_int
        L.moda_attn_decode_noalloc.argtypes = [vp] * 7 + [ctypes.c_int32, sp, vp]
        L.moda_attn_decode_noalloc.restype = ctypes.c_int
        L.moda_attn_decode_noalloc_max_bytes.argtypes = []
        L.moda_attn_decode_noalloc_max_bytes.restype = ctypes.c_size_t
        i32, size, xp = ctypes.c_int32, ctypes.c_size_t, ctypes.POINTER(MODAPrefix)
        L.moda_attn_decode_shared_workspace_bytes.argtypes = [xp, ctypes.c_int, sp]
        L.moda_attn_decode_shared_workspace_bytes.restype = size
        L.moda_attn_decode_shared.argtypes = [vp] * 13 + [i32, vp, size, xp, sp, vp]
        L.moda_attn_decode_shared.restype = ctypes.c_int
        L.moda_attn_decode_weights.argtypes = [vp] * 10 + [i32, vp, size, sp, vp]
        L.moda_attn_decode_weights.restype = ctypes.c_int
        L.moda_attn_weights_workspace_bytes.argtypes = [i32, sp]
        L.moda_attn_weights_workspace_bytes.restype = size
        L.moda_attn_weights.argtypes = [vp] * 6 + [i32, i32, vp, size, sp, vp]
        L.moda_attn_weights.restype = ctypes.c_int
        L.moda_cache_evict_workspace_bytes.argtypes = [i32, sp]
        L.moda_cache_evict_workspace_bytes.restype = size
        L.moda_cache_evict.argtypes = [vp] * 11 + [i32] * 4 + [vp, size, sp, vp]
        L.moda_cache_evict.restype = ctypes.c_int
        gp = ctypes.POINTER(MODAPages)
        L.moda_page_append.argtypes = [vp] * 10 + [gp, sp, vp]
        L.moda_page_append.restype = ctypes.c_int
        L.moda_page_read.argtypes = [vp] * 8 + [i32, gp, sp, vp]
        L.moda_page_read.restype = ctypes.c_int
        L.moda_page_select_workspace_bytes.argtypes = [gp, sp]
        L.moda_page_select_workspace_bytes.restype = size
        L.moda_page_select.argtypes = [vp] * 5 + [i32, i32, i32, vp, size, gp, sp, vp]
        L.moda_page_select.restype = ctypes.c_int
        L.moda_attn_decode_paged_workspace_bytes.argtypes = [gp, sp]
        L.moda_attn_decode_paged_workspace_bytes.restype = size
        L.moda_attn_decode_paged.argtypes = [vp] * 8 + [i32] + [vp] * 5 + [size, gp, sp, vp]
        L.moda_attn_decode_paged.restype = ctypes.c_int
        L.moda_calibrate_mfma_operand_bytes.argtypes = []
        L.moda_calibrate_mfma_operand_bytes.restype = ctypes.c_size_t
        L.moda_calibrate_mfma_sink_bytes.argtypes = [ctypes.c_int32]
        L.moda_calibrate_mfma_sink_bytes.restype = ctypes.c_size_t
        L.moda_calibrate_mfma.argtypes = [vp, vp, ctypes.c_size_t, ctypes.c_int32, ctypes.c_int32, vp]
        L.moda_calibrate_mfma.restype = ctypes.c_double
        L.moda_status_string.argtypes = [ctypes.c_int]
        L.moda_status_string.restype = ctypes.c_char_p
        L.moda_version.restype = ctypes.c_int
        L.moda_kernels_per_call.argtypes = [sp, ctypes.c_int]
        L.moda_kernels_per_call.restype = ctypes.c_int
        L.moda_fwd_kernel_name.argtypes = [sp, ctypes.POINTER(MODAFwdTuning), ctypes.c_char_p, ctypes.c_size_t]
        L.moda_fwd_kernel_name.restype = ctypes.c_int
        L.moda_bwd_kernel_name.argtypes = [sp, ctypes.c_int, ctypes.c_char_p, ctypes.c_size_t]
        L.moda_bwd_kernel_name.restype = ctypes.c_int
        _lib = L
    return _lib


_native_module = None


def _native():
    """Load moda_torch.so and hand it the entry points of libmoda.so.  Raises if absent."""
    global _native_module
    if _native_module is None:
        if not os.path.exists(NATIVE_PATH):
            raise FileNotFoundError(
                "%s not found: build it with `python -m paper_2603_15619_amd.build`" % NATIVE_PATH)
        loader = importlib.machinery.ExtensionFileLoader("moda_torch", NATIVE_PATH)
        m = importlib.util.module_from_spec(importlib.util.spec_from_loader("moda_torch", loader))
        loader.exec_module(m)
        L = lib()
        m.init(*(ctypes.cast(f, ctypes.c_void_p).value for f in
                 (L.moda_attn_fwd, L.moda_attn_bwd, L.moda_attn_bwd_workspace_bytes, L.moda_attn_decode,
                  L.moda_attn_decode_workspace_bytes, L.moda_depth_append)))
        m.init_cache(*(ctypes.cast(f, ctypes.c_void_p).value for f in
                       (L.moda_attn_decode_shared, L.moda_attn_decode_shared_workspace_bytes, L.moda_attn_weights,
                        L.moda_attn_weights_workspace_bytes, L.moda_cache_evict, L.moda_cache_evict_workspace_bytes)))
        m.init_pages(*(ctypes.cast(f, ctypes.c_void_p).value for f in
                       (L.moda_page_append, L.moda_page_read, L.moda_page_select, L.moda_page_select_workspace_bytes,
                        L.moda_attn_decode_paged, L.moda_attn_decode_paged_workspace_bytes)))
        _native_module = m
    return _native_module


def status_string(code: int) -> str:
    return lib().moda_status_string(code).decode()


def _check(code):
    if code != 0:
        raise MODAError(code, status_string(code))


def _outputs(r):
    """What moda_torch returned: the outputs, or the status of a call that the library rejected."""
    if type(r) is int:
        _check(r)
    return r


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _dtype_code(t):
    if t.dtype == torch.bfloat16:
        return MODA_BF16
    if t.dtype == torch.float32:
        return MODA_F32
    raise TypeError("libmoda supports bf16 and fp32 tensors, got %s" % t.dtype)


def make_shape(Q, Kseq, Kdepth, depth_count, causal, scale):
    B, Hq, T, d = Q.shape
    Hk = Kseq.shape[1]
    depth_alloc = 0 if Kdepth is None else Kdepth.shape[3]
    if depth_count is None:
        depth_count = depth_alloc
    return MODAShape(B, Hq, Hk, T, d, depth_alloc, depth_count, int(bool(causal)),
                     float(scale) if scale else 0.0, _dtype_code(Q))


def _require(t, name, shape, dtype, device):
    if t is None:
        return
    if not t.is_cuda:
        raise ValueError("%s must live in device memory" % name)
    if t.device != device or t.dtype != dtype:
        raise ValueError("%s: device/dtype differ from Q" % name)
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s: expected shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)


def _stream(device):
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def moda_attn_fwd(Q, Kseq, Vseq, Kdepth=None, Vdepth=None, depth_count=None, causal=True,
                  scale=None, out=None, lse=None, tuning=None):
    """O, LSE = MoDA attention forward on the current stream of Q's device.

    Q [B,Hq,T,d]; Kseq/Vseq [B,Hk,T,d]; Kdepth/Vdepth [B,Hk,T,depth_alloc,d] or
    None; slots [0, depth_count) of each position are attended (default: all).
    `tuning` = dict(waves=, heads_per_tile=, head_group=, depth_path=) calls moda_attn_fwd_tuned (the bf16
    kernel's launch geometry chosen by the caller; missing keys keep the library's choice).
    """
    if tuning is None:
        r = (_native_module or _native()).fwd(Q, Kseq, Vseq, Kdepth, Vdepth, depth_count, causal, scale, out, lse)
        if r is not None:
            return _outputs(r)
    s = make_shape(Q, Kseq, Kdepth, depth_count, causal, scale)
    dev, dt = Q.device, Q.dtype
    _require(Q, "Q", (s.B, s.Hq, s.T, s.d), dt, dev)
    _require(Kseq, "Kseq", (s.B, s.Hk, s.T, s.d), dt, dev)
    _require(Vseq, "Vseq", (s.B, s.Hk, s.T, s.d), dt, dev)
    _require(Kdepth, "Kdepth", (s.B, s.Hk, s.T, s.depth_alloc, s.d), dt, dev)
    _require(Vdepth, "Vdepth", (s.B, s.Hk, s.T, s.depth_alloc, s.d), dt, dev)
    if out is None:
        out = torch.empty_like(Q)
    if lse is None:
        lse = torch.empty((s.B, s.Hq, s.T), dtype=torch.float32, device=dev)
    _require(out, "out", Q.shape, dt, dev)
    _require(lse, "lse", (s.B, s.Hq, s.T), torch.float32, dev)
    with torch.cuda.device(dev):
        if tuning is None:
            _check(lib().moda_attn_fwd(_ptr(Q), _ptr(Kseq), _ptr(Vseq), _ptr(Kdepth), _ptr(Vdepth),
                                       _ptr(out), _ptr(lse), ctypes.byref(s), _stream(dev)))
        else:
            tn = MODAFwdTuning(int(tuning.get("waves", 0)), int(tuning.get("heads_per_tile", 0)),
                               int(tuning.get("head_group", 0)), int(tuning.get("depth_path", 0)))
            _check(lib().moda_attn_fwd_tuned(_ptr(Q), _ptr(Kseq), _ptr(Vseq), _ptr(Kdepth), _ptr(Vdepth),
                                             _ptr(out), _ptr(lse), ctypes.byref(s), ctypes.byref(tn), _stream(dev)))
    return out, lse


def moda_attn_bwd_workspace_bytes(shape: MODAShape) -> int:
    return int(lib().moda_attn_bwd_workspace_bytes(ctypes.byref(shape)))


def moda_attn_bwd(Q, Kseq, Vseq, Kdepth, Vdepth, O, LSE, dO, depth_count=None, causal=True,
                  scale=None, workspace=None):
    """(dQ, dKseq, dVseq, dKdepth, dVdepth) on the current stream of Q's device."""
    r = (_native_module or _native()).bwd(Q, Kseq, Vseq, Kdepth, Vdepth, O, LSE, dO, depth_count, causal, scale, workspace)
    if r is not None:
        return _outputs(r)
    s = make_shape(Q, Kseq, Kdepth, depth_count, causal, scale)
    dev, dt = Q.device, Q.dtype
    _require(Q, "Q", (s.B, s.Hq, s.T, s.d), dt, dev)
    _require(Kseq, "Kseq", (s.B, s.Hk, s.T, s.d), dt, dev)
    _require(Vseq, "Vseq", (s.B, s.Hk, s.T, s.d), dt, dev)
    _require(Kdepth, "Kdepth", (s.B, s.Hk, s.T, s.depth_alloc, s.d), dt, dev)
    _require(Vdepth, "Vdepth", (s.B, s.Hk, s.T, s.depth_alloc, s.d), dt, dev)
    _require(O, "O", Q.shape, dt, dev)
    _require(dO, "dO", Q.shape, dt, dev)
    _require(LSE, "LSE", (s.B, s.Hq, s.T), torch.float32, dev)
    dQ = torch.empty_like(Q)
    dK = torch.empty_like(Kseq)
    dV = torch.empty_like(Vseq)
    dKd = None if Kdepth is None else torch.empty_like(Kdepth)
    dVd = None if Vdepth is None else torch.empty_like(Vdepth)
    need = moda_attn_bwd_workspace_bytes(s)
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    with torch.cuda.device(dev):
        _check(lib().moda_attn_bwd(_ptr(Q), _ptr(Kseq), _ptr(Vseq), _ptr(Kdepth), _ptr(Vdepth),
                                   _ptr(O), _ptr(LSE), _ptr(dO), _ptr(dQ), _ptr(dK), _ptr(dV),
                                   _ptr(dKd), _ptr(dVd), _ptr(workspace), ws_bytes,
                                   ctypes.byref(s), _stream(dev)))
    return dQ, dK, dV, dKd, dVd


def moda_depth_append(K, V, Kdepth, Vdepth, slot):
    """Depth-stream write step, in place on the current stream: K, V [B,Hk,T,d] become slot
    `slot` of Kdepth, Vdepth [B,Hk,T,depth_alloc,d]."""
    r = (_native_module or _native()).append(K, V, Kdepth, Vdepth, slot)
    if r is not None:
        _outputs(r)
        return Kdepth, Vdepth
    B, Hk, T, d = K.shape
    dev, dt = K.device, K.dtype
    _require(K, "K", (B, Hk, T, d), dt, dev)
    _require(V, "V", (B, Hk, T, d), dt, dev)
    if Kdepth is None or Vdepth is None or Kdepth.dim() != 5:
        raise ValueError("Kdepth / Vdepth: expected [B,Hk,T,depth_alloc,d] tensors")
    La = Kdepth.shape[3]
    _require(Kdepth, "Kdepth", (B, Hk, T, La, d), dt, dev)
    _require(Vdepth, "Vdepth", (B, Hk, T, La, d), dt, dev)
    s = MODAShape(B, Hk, Hk, T, d, La, 0, 1, 0.0, _dtype_code(K))
    with torch.cuda.device(dev):
        _check(lib().moda_depth_append(_ptr(K), _ptr(V), _ptr(Kdepth), _ptr(Vdepth), int(slot),
                                       ctypes.byref(s), _stream(dev)))
    return Kdepth, Vdepth


def moda_attn_decode(Q, Kseq, Vseq, Kdepth=None, Vdepth=None, T=None, depth_count=None, scale=None,
                     out=None, lse=None, workspace=None, noalloc=False):
    """O [B,Hq,d], LSE [B,Hq] for one new token per sequence: Q [B,Hq,d]; sequence cache
    Kseq/Vseq [B,Hk,kv_alloc,d] of which positions [0, T) are attended (default: all); the new
    token's depth slots Kdepth/Vdepth [B,Hk,depth_alloc,d] or None.  noalloc=True calls
    moda_attn_decode_noalloc (the library's own scratch array instead of a workspace; `out`
    and `lse` must then be given, so that this wrapper allocates nothing either)."""
    if not noalloc:
        r = (_native_module or _native()).decode(Q, Kseq, Vseq, Kdepth, Vdepth, T, depth_count, scale, out, lse, workspace)
        if r is not None:
            return _outputs(r)
    B, Hq, d = Q.shape
    Hk, kv_alloc = Kseq.shape[1], Kseq.shape[2]
    T = kv_alloc if T is None else int(T)
    La = 0 if Kdepth is None else Kdepth.shape[2]
    L = La if depth_count is None else int(depth_count)
    dev, dt = Q.device, Q.dtype
    _require(Q, "Q", (B, Hq, d), dt, dev)
    _require(Kseq, "Kseq", (B, Hk, kv_alloc, d), dt, dev)
    _require(Vseq, "Vseq", (B, Hk, kv_alloc, d), dt, dev)
    _require(Kdepth, "Kdepth", (B, Hk, La, d), dt, dev)
    _require(Vdepth, "Vdepth", (B, Hk, La, d), dt, dev)
    s = MODAShape(B, Hq, Hk, T, d, La, L, 1, float(scale) if scale else 0.0, _dtype_code(Q))
    if noalloc and (out is None or lse is None):
        raise ValueError("noalloc=True needs out= and lse=")
    if out is None:
        out = torch.empty_like(Q)
    if lse is None:
        lse = torch.empty((B, Hq), dtype=torch.float32, device=dev)
    _require(out, "out", Q.shape, dt, dev)
    _require(lse, "lse", (B, Hq), torch.float32, dev)
    if noalloc:
        with torch.cuda.device(dev):
            _check(lib().moda_attn_decode_noalloc(_ptr(Q), _ptr(Kseq), _ptr(Vseq), _ptr(Kdepth), _ptr(Vdepth),
                                                  _ptr(out), _ptr(lse), int(kv_alloc), ctypes.byref(s), _stream(dev)))
        return out, lse
    need = int(lib().moda_attn_decode_workspace_bytes(ctypes.byref(s)))
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)
    ws_bytes = workspace.numel() * workspace.element_size()
    with torch.cuda.device(dev):
        _check(lib().moda_attn_decode(_ptr(Q), _ptr(Kseq), _ptr(Vseq), _ptr(Kdepth), _ptr(Vdepth), _ptr(out),
                                      _ptr(lse), int(kv_alloc), _ptr(workspace), ws_bytes, ctypes.byref(s),
                                      _stream(dev)))
    return out, lse


def _workspace(workspace, need, device):
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=device)
    if workspace.device != device or not workspace.is_contiguous():
        raise ValueError("workspace: contiguous tensor on Q's device")
    return workspace, workspace.numel() * workspace.element_size()


def _int32(x, name):
    """int(x), refused where the C ABI's 32 bits do not hold it (ctypes would drop the others)."""
    x = int(x)
    if not -(1 << 31) <= x < 1 << 31:
        raise ValueError("%s: %d does not fit 32 bits" % (name, x))
    return x


def _decode_shared(Q, Kprefix, Vprefix, Kseq, Vseq, Kdepth, Vdepth, prefix_lengths, lengths, P, T, depth_count, scale,
                   weights, weights_out, out, lse, workspace):
    r = (_native_module or _native()).shared(Q, Kprefix, Vprefix, Kseq, Vseq, Kdepth, Vdepth, prefix_lengths, lengths, P, T,
                                             depth_count, scale, weights, weights_out, out, lse, workspace)
    if r is not None:
        return _outputs(r)
    B, Hq, d = Q.shape
    if Kseq is None and Kprefix is None:
        raise ValueError("Kseq or Kprefix must be given")
    Hk = (Kprefix if Kseq is None else Kseq).shape[1]
    kv_alloc = 0 if Kseq is None else Kseq.shape[2]
    T = kv_alloc if T is None else _int32(T, "T")
    La = 0 if Kdepth is None else Kdepth.shape[2]
    L = La if depth_count is None else _int32(depth_count, "depth_count")
    Np, prefix_alloc = (1, 0) if Kprefix is None else (Kprefix.shape[0], Kprefix.shape[2])
    P = prefix_alloc if P is None else _int32(P, "P")
    dev, dt = Q.device, Q.dtype
    _require(Q, "Q", (B, Hq, d), dt, dev)
    _require(Kprefix, "Kprefix", (Np, Hk, prefix_alloc, d), dt, dev)
    _require(Vprefix, "Vprefix", (Np, Hk, prefix_alloc, d), dt, dev)
    _require(Kseq, "Kseq", (B, Hk, kv_alloc, d), dt, dev)
    _require(Vseq, "Vseq", (B, Hk, kv_alloc, d), dt, dev)
    _require(Kdepth, "Kdepth", (B, Hk, La, d), dt, dev)
    _require(Vdepth, "Vdepth", (B, Hk, La, d), dt, dev)
    _require(prefix_lengths, "prefix_lengths", (Np,), torch.int32, dev)
    _require(lengths, "lengths", (B,), torch.int32, dev)
    _require(weights, "weights", (B, Hk, kv_alloc), torch.float32, dev)
    _require(weights_out, "weights_out", (B, Hk, kv_alloc), torch.float32, dev)
    s = MODAShape(B, Hq, Hk, T, d, La, L, 1, float(scale) if scale else 0.0, _dtype_code(Q))
    x = MODAPrefix(Np, P, prefix_alloc)
    if out is None:
        out = torch.empty_like(Q)
    if lse is None:
        lse = torch.empty((B, Hq), dtype=torch.float32, device=dev)
    _require(out, "out", Q.shape, dt, dev)
    _require(lse, "lse", (B, Hq), torch.float32, dev)
    need = 0
    if workspace is None:
        need = int(lib().moda_attn_decode_shared_workspace_bytes(ctypes.byref(x), int(weights_out is not None), ctypes.byref(s)))
    workspace, ws_bytes = _workspace(workspace, need, dev)
    with torch.cuda.device(dev):
        _check(lib().moda_attn_decode_shared(
            _ptr(Q), _ptr(Kprefix), _ptr(Vprefix), _ptr(Kseq), _ptr(Vseq), _ptr(Kdepth), _ptr(Vdepth),
            _ptr(prefix_lengths), _ptr(lengths), _ptr(weights), _ptr(weights_out), _ptr(out), _ptr(lse), kv_alloc,
            _ptr(workspace), ws_bytes, ctypes.byref(x), ctypes.byref(s), _stream(dev)))
    return out, lse


def moda_attn_decode_shared(Q, Kprefix, Vprefix, Kseq, Vseq, Kdepth=None, Vdepth=None, prefix_lengths=None, lengths=None,
                            P=None, T=None, depth_count=None, scale=None, weights=None, weights_out=None, out=None,
                            lse=None, workspace=None):
    """O [B,Hq,d], LSE [B,Hq] for one new token per sequence, under one softmax over the rows of its prefix, of its own
    cache and its depth slots.  Kprefix/Vprefix [n_prefixes,Hk,prefix_alloc,d]: sequence b reads prefix
    b // (B / n_prefixes), whose rows are read once for all that share it.  Kseq/Vseq [B,Hk,kv_alloc,d] (None: no own
    rows), Kdepth/Vdepth [B,Hk,depth_alloc,d] or None.  P and T bound the rows attended (default: all allocated), the int32
    tensors prefix_lengths [n_prefixes] and lengths [B] give them for each.  With weights [B,Hk,kv_alloc] (fp32) the own
    rows' attention weights, summed over the heads of a group, are added to it, in place or, with weights_out, into that."""
    if weights_out is None:
        weights_out = weights
    return _decode_shared(Q, Kprefix, Vprefix, Kseq, Vseq, Kdepth, Vdepth, prefix_lengths, lengths, P, T, depth_count,
                          scale, weights, weights_out, out, lse, workspace)


def moda_attn_decode_weights(Q, Kseq, Vseq, weights=None, Kdepth=None, Vdepth=None, lengths=None, T=None, depth_count=None,
                             scale=None, weights_out=None, out=None, lse=None, workspace=None):
    """O [B,Hq,d], LSE [B,Hq], weights for one new token per sequence: the decoding step over caches of `lengths` [B] rows
    each (default: T), which adds the attention weight of every row, summed over the heads of a group, to
    weights [B,Hk,kv_alloc] (fp32): in place, or into weights_out.  weights None: they start from zero."""
    if weights_out is None:
        weights_out = weights if weights is not None else torch.zeros(Kseq.shape[:3], dtype=torch.float32, device=Q.device)
    out, lse = _decode_shared(Q, None, None, Kseq, Vseq, Kdepth, Vdepth, None, lengths, None, T, depth_count, scale,
                              weights, weights_out, out, lse, workspace)
    return out, lse, weights_out


def moda_attn_weights(Q, Kseq, LSE, window=0, causal=True, scale=None, lengths=None, weights=None, weights_out=None,
                      workspace=None):
    """weights [B,Hk,kv_alloc] (fp32): the attention weight that each row of Kseq [B,Hk,kv_alloc,d] gets from the queries
    Q [B,Hq,T,d] (T <= kv_alloc) whose log-sum-exp LSE [B,Hq,T] the forward pass left, summed over queries and the heads of
    a group; of the last `window` queries only unless that is 0.  lengths [B] (int32): the filled positions of each
    sequence (causal=False: LSE has to leave the others out, which moda_attn_fwd on a padded batch does not).  Added to `weights` where given, in place unless weights_out is."""
    if weights_out is None:
        weights_out = weights if weights is not None else torch.zeros(Kseq.shape[:3], dtype=torch.float32, device=Q.device)
    r = (_native_module or _native()).weights(Q, Kseq, LSE, window, causal, scale, lengths, weights, weights_out, workspace)
    if r is not None:
        _outputs(r)
        return weights_out
    B, Hq, T, d = Q.shape
    Hk, kv_alloc = Kseq.shape[1], Kseq.shape[2]
    window = _int32(window, "window")
    dev, dt = Q.device, Q.dtype
    _require(Q, "Q", (B, Hq, T, d), dt, dev)
    _require(Kseq, "Kseq", (B, Hk, kv_alloc, d), dt, dev)
    _require(LSE, "LSE", (B, Hq, T), torch.float32, dev)
    _require(lengths, "lengths", (B,), torch.int32, dev)
    _require(weights, "weights", (B, Hk, kv_alloc), torch.float32, dev)
    _require(weights_out, "weights_out", (B, Hk, kv_alloc), torch.float32, dev)
    s = MODAShape(B, Hq, Hk, T, d, 0, 0, int(bool(causal)), float(scale) if scale else 0.0, _dtype_code(Q))
    need = int(lib().moda_attn_weights_workspace_bytes(window, ctypes.byref(s))) if workspace is None else 0
    workspace, ws_bytes = _workspace(workspace, need, dev)
    with torch.cuda.device(dev):
        _check(lib().moda_attn_weights(_ptr(Q), _ptr(Kseq), _ptr(LSE), _ptr(lengths), _ptr(weights), _ptr(weights_out),
                                       window, kv_alloc, _ptr(workspace), ws_bytes, ctypes.byref(s), _stream(dev)))
    return weights_out


def moda_cache_evict(Kseq, Vseq, weights, keep, recent=0, positions=None, lengths=None, T=None, out=None, lengths_out=None,
                     index=None, workspace=None):
    """index [B,Hk,min(keep,T)], lengths [B] (both int32): each (sequence, key/value head) keeps its `recent` newest rows and
    the heaviest others, `keep` in all.  Kseq/Vseq [B,Hk,kv_alloc,d], weights [B,Hk,kv_alloc] (fp32), positions
    [B,Hk,kv_alloc] (int32, the rows' token positions; None: their row numbers), of which lengths [B] (None: T, None: all)
    rows are filled.  The kept rows end up in rows [0, new length): in place, or, with out = (Kout, Vout, weights_out,
    positions_out or None) of out_alloc >= min(keep, T) rows, there.  index: the row that each came from, -1 behind them.
    Without lengths_out a call in place overwrites `lengths`, if given; else the new lengths are a new tensor."""
    B, Hk, kv_alloc, d = Kseq.shape
    T = kv_alloc if T is None else _int32(T, "T")
    keep = _int32(keep, "keep")
    n = max(0, min(keep, T))
    dev, dt = Kseq.device, Kseq.dtype
    Kout, Vout, W_out, P_out = (Kseq, Vseq, weights, positions) if out is None else out
    if Kout.dim() != 4:
        raise ValueError("Kout: expected a [B,Hk,out_alloc,d] tensor")
    out_alloc = Kout.shape[2]
    if lengths_out is None:
        lengths_out = lengths if lengths is not None and out is None else torch.empty(B, dtype=torch.int32, device=dev)
    if index is None:
        index = torch.empty((B, Hk, n), dtype=torch.int32, device=dev)
    r = (_native_module or _native()).evict(Kseq, Vseq, weights, positions, lengths, Kout, Vout, W_out, P_out, lengths_out, index,
                                            keep, recent, T, workspace)
    if r is not None:
        _outputs(r)
        return index, lengths_out
    recent = _int32(recent, "recent")
    _require(Kseq, "Kseq", (B, Hk, kv_alloc, d), dt, dev)
    _require(Vseq, "Vseq", (B, Hk, kv_alloc, d), dt, dev)
    _require(weights, "weights", (B, Hk, kv_alloc), torch.float32, dev)
    _require(positions, "positions", (B, Hk, kv_alloc), torch.int32, dev)
    _require(lengths, "lengths", (B,), torch.int32, dev)
    _require(Kout, "Kout", (B, Hk, out_alloc, d), dt, dev)
    _require(Vout, "Vout", (B, Hk, out_alloc, d), dt, dev)
    _require(W_out, "weights_out", (B, Hk, out_alloc), torch.float32, dev)
    _require(P_out, "positions_out", (B, Hk, out_alloc), torch.int32, dev)
    _require(lengths_out, "lengths_out", (B,), torch.int32, dev)
    _require(index, "index", (B, Hk, n), torch.int32, dev)
    s = MODAShape(B, Hk, Hk, T, d, 0, 0, 1, 0.0, _dtype_code(Kseq))
    need = int(lib().moda_cache_evict_workspace_bytes(keep, ctypes.byref(s))) if workspace is None else 0
    workspace, ws_bytes = _workspace(workspace, need, dev)
    with torch.cuda.device(dev):
        _check(lib().moda_cache_evict(
            _ptr(Kseq), _ptr(Vseq), _ptr(weights), _ptr(positions), _ptr(lengths), _ptr(Kout), _ptr(Vout), _ptr(W_out),
            _ptr(P_out), _ptr(lengths_out), _ptr(index), keep, recent, kv_alloc, out_alloc, _ptr(workspace), ws_bytes,
            ctypes.byref(s), _stream(dev)))
    return index, lengths_out


def _pages(Kpages, Vpages, page_table, Kscales, Vscales, B, device):
    """The pools' shape, MODAPages and (n_pages, Hk, page_rows, d): bf16 pools without scales, or e4m3 pools with both."""
    if Kpages.dim() != 4 or page_table.dim() != 2:
        raise ValueError("expected Kpages [n_pages,Hk,page_rows,d] and page_table [B,max_pages]")
    n, Hk, R, d = Kpages.shape
    mx = Kpages.dtype == torch.float8_e4m3fn
    if not mx and Kpages.dtype != torch.bfloat16:
        raise TypeError("pages hold bf16 or float8_e4m3fn, got %s" % Kpages.dtype)
    if mx != (Kscales is not None) or mx != (Vscales is not None):
        raise ValueError("Kscales and Vscales belong to float8_e4m3fn pages, and to them only")
    max_pages = page_table.shape[1]
    _require(Kpages, "Kpages", (n, Hk, R, d), Kpages.dtype, device)
    _require(Vpages, "Vpages", (n, Hk, R, d), Kpages.dtype, device)
    _require(Kscales, "Kscales", (n, Hk, R, d // 32), torch.uint8, device)
    _require(Vscales, "Vscales", (n, Hk, R, d // 32), torch.uint8, device)
    _require(page_table, "page_table", (B, max_pages), torch.int32, device)
    return MODAPages(_int32(n, "n_pages"), _int32(R, "page_rows"), _int32(max_pages, "max_pages"), MODA_PAGES_MX8 if mx else MODA_PAGES_BF16)


def _bound(T, page_table, page_rows):
    """Rows that lengths may reach: T, or (None) all that the table has."""
    return _int32(page_table.shape[1] * page_rows if T is None else T, "T")


def moda_page_append(K, V, Kpages, Vpages, page_table, lengths=None, counts=None, Kscales=None, Vscales=None, Kbounds=None):
    """New rows K, V [B,Hk,T,d] go to their places in the pages of a paged cache, in place: Kpages/Vpages [n_pages,Hk,page_rows,d] in
    bf16, or in float8_e4m3fn with Kscales/Vscales [n_pages,Hk,page_rows,d/32] (uint8 exponents + 127); page_table [B,max_pages]
    (int32): the page of each page_rows rows of a sequence, -1: none.  lengths [B] (int32; None: T): the rows of each sequence after
    the call, of which the last min(T, counts [B], length) are the new ones.  Kbounds [n_pages,Hk,2,d] (bf16): the least and
    largest key channels of every page written are kept there.  Returns Kpages, Vpages."""
    r = (_native_module or _native()).page_append(K, V, Kpages, Vpages, page_table, lengths, counts, Kscales, Vscales, Kbounds)
    if r is not None:
        _outputs(r)
        return Kpages, Vpages
    B, Hk, T, d = K.shape
    dev = K.device
    x = _pages(Kpages, Vpages, page_table, Kscales, Vscales, B, dev)
    if Kpages.shape[1] != Hk or Kpages.shape[3] != d:
        raise ValueError("Kpages: expected %d heads of dimension %d, got %s" % (Hk, d, tuple(Kpages.shape)))
    _require(K, "K", (B, Hk, T, d), torch.bfloat16, dev)
    _require(V, "V", (B, Hk, T, d), torch.bfloat16, dev)
    _require(lengths, "lengths", (B,), torch.int32, dev)
    _require(counts, "counts", (B,), torch.int32, dev)
    _require(Kbounds, "Kbounds", (x.n_pages, Hk, 2, d), torch.bfloat16, dev)
    s = MODAShape(B, Hk, Hk, _int32(T, "T"), d, 0, 0, 1, 0.0, MODA_BF16)
    with torch.cuda.device(dev):
        _check(lib().moda_page_append(_ptr(K), _ptr(V), _ptr(page_table), _ptr(lengths), _ptr(counts), _ptr(Kpages), _ptr(Vpages),
                                      _ptr(Kscales), _ptr(Vscales), _ptr(Kbounds), ctypes.byref(x), ctypes.byref(s), _stream(dev)))
    return Kpages, Vpages


def moda_page_read(Kpages, Vpages, page_table, lengths=None, first=0, T=None, Kscales=None, Vscales=None, out=None):
    """K, V [B,Hk,T,d] (bf16): rows [first, first + T) of every sequence of a paged cache (moda_page_append has its arguments), exactly as the
    pages hold them.  T None: that of `out`, else all rows that the table has from `first` on.  Rows from a sequence's
    length on (lengths [B]; None: all are there) and those of missing pages are left as they were in out = (K, V); without
    `out` they are zero."""
    if out is not None and T is None:
        r = (_native_module or _native()).page_read(Kpages, Vpages, page_table, lengths, first, Kscales, Vscales, *out)
        if r is not None:
            _outputs(r)
            return out[0], out[1]
    B, dev = page_table.shape[0], Kpages.device
    x = _pages(Kpages, Vpages, page_table, Kscales, Vscales, B, dev)
    Hk, d = Kpages.shape[1], Kpages.shape[3]
    first = _int32(first, "first")
    if T is None:
        T = out[0].shape[2] if out is not None else max(0, x.max_pages * x.page_rows - first)
    T = _int32(T, "T")
    if T < 0:
        raise ValueError("T: %d rows" % T)
    if out is None:
        out = tuple(torch.zeros((B, Hk, T, d), dtype=torch.bfloat16, device=dev) for _ in range(2))
    K, V = out
    _require(K, "K", (B, Hk, T, d), torch.bfloat16, dev)
    _require(V, "V", (B, Hk, T, d), torch.bfloat16, dev)
    _require(lengths, "lengths", (B,), torch.int32, dev)
    s = MODAShape(B, Hk, Hk, T, d, 0, 0, 1, 0.0, MODA_BF16)
    with torch.cuda.device(dev):
        _check(lib().moda_page_read(_ptr(Kpages), _ptr(Vpages), _ptr(Kscales), _ptr(Vscales), _ptr(page_table), _ptr(lengths), _ptr(K),
                                    _ptr(V), first, ctypes.byref(x), ctypes.byref(s), _stream(dev)))
    return K, V


def moda_page_select(Q, Kbounds, page_table, keep, page_rows, lengths=None, first=1, recent=1, T=None, out=None, workspace=None):
    """pages [B,Hk,keep] (int32): for each (sequence, key/value head) the `first` first and `recent` last pages and those whose key bounds
    Kbounds [n_pages,Hk,2,d] promise the largest logits, summed over the heads of the group, for the queries Q [B,Hq,d]; indices into
    the sequence's row of page_table [B,max_pages], ascending, -1 behind the last.  lengths [B] (int32; None: T, None: all rows that the
    table has); T bounds them, and decides the kernels and the workspace.  What moda_attn_decode_paged takes as `selected`."""
    if out is not None:
        r = (_native_module or _native()).page_select(Q, Kbounds, page_table, keep, page_rows, lengths, first, recent, T, out, workspace)
        if r is not None:
            _outputs(r)
            return out
    B, Hq, d = Q.shape
    dev = Q.device
    if Kbounds.dim() != 4 or page_table.dim() != 2:
        raise ValueError("expected Kbounds [n_pages,Hk,2,d] and page_table [B,max_pages]")
    n, Hk, max_pages = Kbounds.shape[0], Kbounds.shape[1], page_table.shape[1]
    keep, first, recent, page_rows = _int32(keep, "keep"), _int32(first, "first"), _int32(recent, "recent"), _int32(page_rows, "page_rows")
    T = _bound(T, page_table, page_rows)
    _require(Q, "Q", (B, Hq, d), torch.bfloat16, dev)
    _require(Kbounds, "Kbounds", (n, Hk, 2, d), torch.bfloat16, dev)
    _require(page_table, "page_table", (B, max_pages), torch.int32, dev)
    _require(lengths, "lengths", (B,), torch.int32, dev)
    if out is None:
        out = torch.empty((B, Hk, max(keep, 0)), dtype=torch.int32, device=dev)
    _require(out, "out", (B, Hk, keep), torch.int32, dev)
    x = MODAPages(_int32(n, "n_pages"), page_rows, _int32(max_pages, "max_pages"), MODA_PAGES_BF16)
    s = MODAShape(B, Hq, Hk, T, d, 0, 0, 1, 0.0, MODA_BF16)
    need = int(lib().moda_page_select_workspace_bytes(ctypes.byref(x), ctypes.byref(s))) if workspace is None else 0
    workspace, ws_bytes = _workspace(workspace, need, dev)
    with torch.cuda.device(dev):
        _check(lib().moda_page_select(_ptr(Q), _ptr(Kbounds), _ptr(page_table), _ptr(lengths), _ptr(out), keep, first, recent,
                                      _ptr(workspace), ws_bytes, ctypes.byref(x), ctypes.byref(s), _stream(dev)))
    return out


def moda_attn_decode_paged(Q, Kpages, Vpages, page_table, Kdepth=None, Vdepth=None, lengths=None, selected=None, Kscales=None,
                           Vscales=None, T=None, depth_count=None, scale=None, out=None, lse=None, workspace=None):
    """O [B,Hq,d], LSE [B,Hq] for one new token per sequence, under one softmax over the rows of its pages (moda_page_append has
    the cache's arguments; the token's own row is among them) and its depth slots Kdepth/Vdepth [B,Hk,depth_alloc,d] or None.
    lengths [B] (int32): the rows of each sequence; T bounds them (default: all rows that the table has) and is their number where lengths is
    None.  T also decides the kernels: under a table much wider than the sequences, a T of the longest length that may come is faster.
    selected [B,Hk,n] (int32): only the rows of these pages, indices into the sequence's row of page_table, each once, -1: none."""
    r = (_native_module or _native()).paged(Q, Kpages, Vpages, page_table, Kdepth, Vdepth, lengths, selected, Kscales, Vscales, T,
                                            depth_count, scale, out, lse, workspace)
    if r is not None:
        return _outputs(r)
    B, Hq, d = Q.shape
    dev = Q.device
    x = _pages(Kpages, Vpages, page_table, Kscales, Vscales, B, dev)
    Hk = Kpages.shape[1]
    if Kpages.shape[3] != d:
        raise ValueError("Kpages: expected a head dimension of %d, got %s" % (d, tuple(Kpages.shape)))
    T = _bound(T, page_table, x.page_rows)
    La = 0 if Kdepth is None else Kdepth.shape[2]
    L = La if depth_count is None else _int32(depth_count, "depth_count")
    _require(Q, "Q", (B, Hq, d), torch.bfloat16, dev)
    _require(Kdepth, "Kdepth", (B, Hk, La, d), torch.bfloat16, dev)
    _require(Vdepth, "Vdepth", (B, Hk, La, d), torch.bfloat16, dev)
    _require(lengths, "lengths", (B,), torch.int32, dev)
    n_selected = 0
    if selected is not None:
        if selected.dim() != 3 or selected.shape[2] == 0:
            raise ValueError("selected: expected a [B,Hk,n] tensor, n > 0")
        n_selected = _int32(selected.shape[2], "n_selected")
        _require(selected, "selected", (B, Hk, n_selected), torch.int32, dev)
    if out is None:
        out = torch.empty_like(Q)
    if lse is None:
        lse = torch.empty((B, Hq), dtype=torch.float32, device=dev)
    _require(out, "out", Q.shape, torch.bfloat16, dev)
    _require(lse, "lse", (B, Hq), torch.float32, dev)
    s = MODAShape(B, Hq, Hk, T, d, La, L, 1, float(scale) if scale else 0.0, MODA_BF16)
    need = int(lib().moda_attn_decode_paged_workspace_bytes(ctypes.byref(x), ctypes.byref(s))) if workspace is None else 0
    workspace, ws_bytes = _workspace(workspace, need, dev)
    with torch.cuda.device(dev):
        _check(lib().moda_attn_decode_paged(
            _ptr(Q), _ptr(Kpages), _ptr(Vpages), _ptr(Kscales), _ptr(Vscales), _ptr(page_table), _ptr(lengths), _ptr(selected), n_selected,
            _ptr(Kdepth), _ptr(Vdepth), _ptr(out), _ptr(lse), _ptr(workspace), ws_bytes, ctypes.byref(x), ctypes.byref(s), _stream(dev)))
    return out, lse


def moda_calibrate_mfma(operands, workgroups, iters, sink=None):
    """Enqueue the matrix-pipe calibration kernel on the current stream; returns the floating-point
    operations of the launch.  `operands`: bf16 tensor of moda_calibrate_mfma_operand_bytes() bytes."""
    dev = operands.device
    need = int(lib().moda_calibrate_mfma_operand_bytes())
    if operands.dtype != torch.bfloat16 or operands.numel() * 2 < need or not operands.is_contiguous():
        raise ValueError("operands: contiguous bf16 tensor of at least %d bytes" % need)
    sb = int(lib().moda_calibrate_mfma_sink_bytes(int(workgroups)))
    if sink is None:
        sink = torch.empty(sb // 4, dtype=torch.float32, device=dev)
    with torch.cuda.device(dev):
        fl = float(lib().moda_calibrate_mfma(_ptr(operands), _ptr(sink), sink.numel() * 4, int(workgroups), int(iters),
                                             _stream(dev)))
    if fl <= 0:
        raise MODAError(5, "calibration launch rejected")
    return fl
