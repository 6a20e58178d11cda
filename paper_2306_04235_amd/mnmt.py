"""Thin Python binding of libmnmt (the C ABI in include/mnmt.h).

Argument marshalling only: every step of inference runs in the library's HIP
kernels.  PyTorch provides device memory (the model arena and the session
workspace are torch uint8 tensors) and streams.  There is no fallback: if the
library is not built, ``lib()`` raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmnmt.so")

OK, E_INVALID_ARG, E_BAD_MODEL, E_CAPACITY, E_HIP, E_UNSUPPORTED, E_TIMEOUT = 0, -1, -2, -3, -4, -5, -6
(EPI_I32, EPI_I8, EPI_I8_RELU, EPI_F32, EPI_F32_RESID, EPI_LOGITS, EPI_ARGMAX, EPI_ARGMAX_PARTIAL,
 EPI_ARGMAX_PARTIAL_PACKED) = range(9)

LOAD_PACKED_4BIT_ONLY = 1

ATTN_I8, ATTN_F32 = 0, 1

EXPORTS = ("mnmt_model_bytes", "mnmt_model_load", "mnmt_model_bytes_ex", "mnmt_model_load_ex", "mnmt_model_get_info", "mnmt_model_free", "mnmt_session_bytes",
           "mnmt_session_create", "mnmt_session_free", "mnmt_encode", "mnmt_decode_step", "mnmt_translate",
           "mnmt_session_status", "mnmt_session_tensor", "mnmt_qlinear", "mnmt_qlinear_w4", "mnmt_qlinear_timed",
           "mnmt_argmax_partials", "mnmt_packed_bytes", "mnmt_pack_weights", "mnmt_logits_argmax_noalloc",
           "mnmt_pages_bytes", "mnmt_pages_ws_bytes", "mnmt_pages_fork", "mnmt_pages_compact", "mnmt_pages_write",
           "mnmt_attn_ws_bytes", "mnmt_attn_paged", "mnmt_attn_cross",
           "mnmt_fold_requant", "mnmt_debug_canon", "mnmt_debug_read", "mnmt_status_str", "mnmt_last_error")


class MnmtError(RuntimeError):
    def __init__(self, status: int, where: str):
        msg = lib().mnmt_last_error().decode(errors="replace")
        super().__init__(f"{where}: {lib().mnmt_status_str(status).decode()} ({status}): {msg}")
        self.status = status


class ModelInfo(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("d_model", "n_heads", "d_ffn", "n_enc", "n_dec", "vocab", "max_pos",
                                         "ln_post", "pad_id", "bos_id", "eos_id", "unk_id")] + [
        ("ln_eps", C.c_float), ("emb_dim", C.c_int32)]


class SessionCfg(C.Structure):
    _fields_ = [("max_batch", C.c_int32), ("max_src_len", C.c_int32), ("max_tgt_len", C.c_int32),
                ("beam", C.c_int32)]


class SearchCfg(C.Structure):
    _fields_ = [("beam", C.c_int32), ("max_steps", C.c_int32), ("len_penalty_alpha", C.c_float),
                ("stop_at_eos", C.c_int32), ("use_graph", C.c_int32)]


class PagesCfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "n_pages", "page_size", "n_kv_heads", "d_head", "max_pages")]


class AttnCfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_heads", "kind", "causal", "ld_q", "ld_out", "max_q", "max_len")] + [
        ("c_qk", C.c_float), ("c_pv", C.c_float)]


_lib = None


def lib():
    """Load libmnmt.so; raises if it has not been built (no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                               "or python paper_2306_04235_amd/build.py")
        L = C.CDLL(LIB_PATH)
        vp, sz, i32, f32 = C.c_void_p, C.c_size_t, C.c_int, C.c_float
        L.mnmt_model_bytes.argtypes = [C.c_char_p, sz, C.POINTER(sz)]
        L.mnmt_model_load.argtypes = [C.c_char_p, sz, vp, sz, vp, C.POINTER(vp)]
        L.mnmt_model_bytes_ex.argtypes = [C.c_char_p, sz, C.c_uint, C.POINTER(sz)]
        L.mnmt_model_load_ex.argtypes = [C.c_char_p, sz, C.c_uint, vp, sz, vp, C.POINTER(vp)]
        L.mnmt_model_get_info.argtypes = [vp, C.POINTER(ModelInfo)]
        L.mnmt_model_free.argtypes = [vp]
        L.mnmt_model_free.restype = None
        L.mnmt_session_bytes.argtypes = [vp, C.POINTER(SessionCfg), C.POINTER(sz)]
        L.mnmt_session_create.argtypes = [vp, C.POINTER(SessionCfg), vp, sz, C.POINTER(vp)]
        L.mnmt_session_free.argtypes = [vp]
        L.mnmt_session_free.restype = None
        L.mnmt_encode.argtypes = [vp, vp, vp, i32, i32, vp]
        L.mnmt_decode_step.argtypes = [vp, vp, vp, vp, vp]
        L.mnmt_translate.argtypes = [vp, vp, vp, i32, i32, C.POINTER(SearchCfg), vp, vp, vp, vp]
        L.mnmt_session_tensor.argtypes = [vp, C.c_char_p, C.POINTER(vp), C.POINTER(sz)]
        L.mnmt_session_status.argtypes = [vp, vp]
        L.mnmt_qlinear.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, f32, vp, vp]
        L.mnmt_qlinear_w4.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, f32, vp, vp]
        L.mnmt_qlinear_timed.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, f32, vp, vp, vp, vp]
        L.mnmt_argmax_partials.argtypes = [i32]
        L.mnmt_packed_bytes.argtypes = [i32, i32]
        L.mnmt_packed_bytes.restype = sz
        L.mnmt_pack_weights.argtypes = [vp, i32, i32, vp, vp]
        L.mnmt_fold_requant.argtypes = [f32, vp, vp, f32, i32, vp, vp]
        L.mnmt_debug_canon.argtypes = [i32, vp, i32, vp, vp]
        L.mnmt_debug_read.argtypes = [vp, sz, i32, vp, vp]
        L.mnmt_logits_argmax_noalloc.argtypes = [vp, vp, vp, i32, i32, i32, vp, vp, vp]
        i64, pages, attn = C.c_int64, C.POINTER(PagesCfg), C.POINTER(AttnCfg)
        L.mnmt_pages_bytes.argtypes = [pages]
        L.mnmt_pages_bytes.restype = sz
        L.mnmt_pages_ws_bytes.argtypes = [pages, i32]
        L.mnmt_pages_ws_bytes.restype = sz
        L.mnmt_pages_fork.argtypes = [pages, vp, vp, vp, i32, vp, vp, i32, vp, vp, vp, vp, sz, vp]
        L.mnmt_pages_compact.argtypes = [pages, vp, vp, vp, i32, vp, vp, vp, sz, vp]
        L.mnmt_pages_write.argtypes = [pages, vp, i32, vp, vp, i32, vp, vp, i64, vp, i32, i32, vp]
        L.mnmt_attn_ws_bytes.argtypes = [i32] * 7
        L.mnmt_attn_ws_bytes.restype = sz
        L.mnmt_attn_paged.argtypes = [pages, attn, vp, i32, vp, vp, i32, vp, vp, i32, vp, vp, sz, vp]
        L.mnmt_attn_cross.argtypes = [attn, i32, i32, vp, vp, i64, i64, i32, vp, i32, vp, vp, i32, vp, vp, sz, vp]
        L.mnmt_status_str.argtypes = [i32]
        L.mnmt_status_str.restype = C.c_char_p
        L.mnmt_last_error.argtypes = []
        L.mnmt_last_error.restype = C.c_char_p
        _lib = L
    return _lib


def _check(rc: int, where: str):
    if rc != OK:
        raise MnmtError(rc, where)


def _ptr(t):
    """A tensor's address (ctypes takes an int or None as void*; a c_void_p
    object per argument costs more than the call's own checks)."""
    return None if t is None else t.data_ptr()


_raw_stream = None


def _stream(stream=None):
    """The stream's hipStream_t as an int: the given one, or the current one of
    the current device."""
    if stream is not None:
        return stream.cuda_stream
    global _raw_stream
    if _raw_stream is None:
        import torch

        # torch.cuda.current_stream() builds a Stream object around this value
        # (2 us of an 8 us call); the raw accessor is what it is built from
        raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        if raw is not None and device is not None:
            torch.cuda.current_stream()  # (the first call initializes the runtime)
            _raw_stream = lambda: raw(device())  # noqa: E731
        else:
            _raw_stream = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
    return _raw_stream()


# ---- host-only entry points ---------------------------------------------------
def mnmt_model_bytes(blob: bytes, flags: int = 0) -> int:
    n = C.c_size_t()
    _check(lib().mnmt_model_bytes_ex(blob, len(blob), flags, C.byref(n)), "mnmt_model_bytes_ex")
    return n.value


def mnmt_fold_requant(s_in, s_w, b, s_out):
    import numpy as np

    s_w = np.ascontiguousarray(s_w, np.float32)
    b = np.ascontiguousarray(b, np.float32)
    sc, bi = np.empty_like(s_w), np.empty_like(s_w)
    _check(lib().mnmt_fold_requant(float(s_in), s_w.ctypes.data, b.ctypes.data, float(s_out), s_w.size,
                                   sc.ctypes.data, bi.ctypes.data), "mnmt_fold_requant")
    return sc, bi


# ---- device entry points ---------------------------------------------------------
def _linear_out(X, M, N, epilogue):
    """A new output tensor for the epilogue."""
    import torch

    if epilogue == EPI_ARGMAX:
        return torch.zeros(M, dtype=torch.int64, device=X.device)  # packed (key, index) per row
    if epilogue in (EPI_ARGMAX_PARTIAL, EPI_ARGMAX_PARTIAL_PACKED):
        return torch.empty((M, argmax_partials(N)), dtype=torch.int64, device=X.device)
    dt = torch.int32 if epilogue == EPI_I32 else torch.int8 if epilogue in (EPI_I8, EPI_I8_RELU) else torch.float32
    return torch.empty((M, N), dtype=dt, device=X.device)


def mnmt_qlinear(X, W, scale, bias, epilogue, gamma=1.0, out=None, stream=None, n_out=None):
    """Y = epilogue(X W^T) for int8 CUDA tensors X [M, K], W [N, K] (for
    EPI_ARGMAX_PARTIAL_PACKED, W is mnmt_pack_weights' output and n_out = N)."""
    M, K = X.shape
    N = W.shape[0] if n_out is None else int(n_out)
    if out is None:
        out = _linear_out(X, M, N, epilogue)
    rc = (_lib or lib()).mnmt_qlinear(_ptr(X), _ptr(W), _ptr(scale), _ptr(bias), M, K, N, epilogue, float(gamma),
                                      _ptr(out), _stream(stream))
    if rc:
        _check(rc, "mnmt_qlinear")
    return out


def mnmt_qlinear_w4(X, W4, scale, bias, epilogue, gamma=1.0, out=None, stream=None):
    """Y = epilogue(X W^T) for int8 CUDA tensor X [M, K] and W's packed 4-bit
    rows W4 uint8 [N, K / 2] (the model file's format)."""
    M, K = X.shape
    N = W4.shape[0]
    if out is None:
        import torch

        dt = torch.int32 if epilogue == EPI_I32 else torch.int8 if epilogue in (EPI_I8, EPI_I8_RELU) else torch.float32
        out = torch.empty((M, N), dtype=dt, device=X.device)
    rc = (_lib or lib()).mnmt_qlinear_w4(_ptr(X), _ptr(W4), _ptr(scale), _ptr(bias), M, K, N, epilogue,
                                         float(gamma), _ptr(out), _stream(stream))
    if rc:
        _check(rc, "mnmt_qlinear_w4")
    return out


def mnmt_qlinear_timed(X, W, scale, bias, epilogue, ev_start, ev_stop, gamma=1.0, out=None, stream=None,
                       n_out=None):
    """mnmt_qlinear bracketed by two torch.cuda.Event(enable_timing=True)
    (recorded once beforehand so that their HIP events exist)."""
    import torch

    M, K = X.shape
    N = W.shape[0] if n_out is None else int(n_out)
    if out is None:
        partial = epilogue in (EPI_ARGMAX_PARTIAL, EPI_ARGMAX_PARTIAL_PACKED)
        shape = (M, argmax_partials(N)) if partial else (M,)
        out = torch.zeros(shape, dtype=torch.int64, device=X.device)
    _check(lib().mnmt_qlinear_timed(_ptr(X), _ptr(W), _ptr(scale), _ptr(bias), M, K, N, epilogue, float(gamma),
                                    _ptr(out), _stream(stream), C.c_void_p(ev_start.cuda_event),
                                    C.c_void_p(ev_stop.cuda_event)), "mnmt_qlinear_timed")
    return out


def mnmt_pack_weights(W, stream=None):
    """Fragment-order copy of an int8 CUDA tensor W [N, K] (K a multiple of
    64): an int8 tensor [ceil(N / 16) * 16, K] whose bytes are in the order
    mnmt_pack_weights documents (not a row-major matrix)."""
    import torch

    N, K = W.shape
    if W.dtype != torch.int8 or not W.is_contiguous():
        raise ValueError("W must be a contiguous int8 tensor")
    nbytes = lib().mnmt_packed_bytes(int(N), int(K))
    if nbytes == 0:
        raise ValueError(f"cannot pack a [{N}, {K}] weight (K must be a positive multiple of 64)")
    out = torch.empty((nbytes // K, K), dtype=torch.int8, device=W.device)
    _check(lib().mnmt_pack_weights(_ptr(W), int(N), int(K), _ptr(out), _stream(stream)), "mnmt_pack_weights")
    return out


def argmax_partials(N: int) -> int:
    """Partial keys per row of an MNMT_EPI_ARGMAX_PARTIAL result for N outputs."""
    p = lib().mnmt_argmax_partials(int(N))
    if p < 1:
        raise ValueError(f"no arg-max partials for N={N}")
    return p


def argmax_index(packed):
    """Vocabulary index held in an MNMT_EPI_ARGMAX result (int64 tensor or array)."""
    import numpy as np

    low = np.asarray(packed.cpu() if hasattr(packed, "cpu") else packed).astype(np.int64) & 0xFFFFFFFF
    return (0xFFFFFFFF - low).astype(np.int64)


def mnmt_debug_canon(fn: int, x, stream=None):
    import torch

    y = torch.empty(x.numel() if fn != 2 else 1, dtype=torch.float32, device=x.device)
    _check(lib().mnmt_debug_canon(fn, _ptr(x), x.numel(), _ptr(y), _stream(stream)), "mnmt_debug_canon")
    return y


def mnmt_logits_argmax_noalloc(X, Wp, scale, N, key=None, tok=None, stream=None):
    """Per-row arg-max key (int64 view of the uint64) and index of X [M, K] against
    the packed weight Wp (mnmt_pack_weights), with no caller scratch."""
    import torch

    M, K = X.shape
    if key is None:
        key = torch.empty(M, dtype=torch.int64, device=X.device)
    if tok is None:
        tok = torch.empty(M, dtype=torch.int32, device=X.device)
    _check(lib().mnmt_logits_argmax_noalloc(_ptr(X), _ptr(Wp), _ptr(scale), M, K, N, _ptr(key), _ptr(tok),
                                            _stream(stream)), "mnmt_logits_argmax_noalloc")
    return key, tok


DEBUG_READ_BLOCKS = 2048


def mnmt_debug_read(x, sink, reps=1, stream=None):
    """Read every byte of the device tensor x `reps` times (bandwidth probe); sink: int32 [2048]."""
    if sink.numel() * sink.element_size() < 4 * DEBUG_READ_BLOCKS:
        raise ValueError("sink needs 2048 32-bit words")
    _check(lib().mnmt_debug_read(_ptr(x), x.numel() * x.element_size(), int(reps), _ptr(sink), _stream(stream)),
           "mnmt_debug_read")


# ---- paged cache and attention ---------------------------------------------------------
@functools.lru_cache(maxsize=256)
def _pages(pool_shape, width: int, rows: int):
    """A pool's configuration (as the C ABI takes it) and the workspace of a fork or compaction of `rows` rows."""
    _need(len(pool_shape) == 6 and pool_shape[2] == 2,
          "the pool must be a contiguous int8 tensor [n_layers, n_pages, 2, n_kv_heads, page_size, d_head]")
    L, n, _, hkv, P, dh = pool_shape
    cfg = PagesCfg(L, n, P, hkv, dh, width)
    return cfg, C.byref(cfg), lib().mnmt_pages_ws_bytes(C.byref(cfg), rows)


@functools.lru_cache(maxsize=256)
def _attn(rows, n, hkv, dh, d, kind, causal, ld, ldo, most, longest, c_qk, c_pv):
    """An attention call's configuration and workspace.  (Plain numbers all: a tensor would be known by its identity.)"""
    _need(dh > 0 and d > 0 and d % dh == 0, "q must have whole heads")
    # (ctypes would take such a number's low bits)
    _need(max(rows, n, d, ld, ldo, most, longest) < 1 << 31, "sizes and strides must be below 2^31")
    a = AttnCfg(d // dh, kind, causal, ld, ldo, most, longest, c_qk, c_pv)
    return C.byref(a), lib().mnmt_attn_ws_bytes(rows, n, d // dh, hkv, dh, most, longest)


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _pool(pool, width, rows):
    _need(pool.dtype is _int8 and pool.is_contiguous(),
          "the pool must be a contiguous int8 tensor [n_layers, n_pages, 2, n_kv_heads, page_size, d_head]")
    return _pages(pool.shape, width, rows)


def _ints(name, t, shape, device):
    """Checks an int32 tensor that the kernels read as a dense array."""
    if t.dtype is not _int32 or t.shape != shape or not t.is_contiguous() or t.get_device() != device:
        raise ValueError(f"{name} must be a contiguous int32 tensor {list(shape)} on device {device}")


def _codes(name, t, width, device):
    """Checks int8 rows [n, width] whose columns are adjacent; their stride."""
    n, w = t.shape
    stride, one = t.stride()
    if t.dtype is not _int8 or w != width or (one != 1 and n and w) or t.get_device() != device:
        raise ValueError(f"{name} must be int8 [n, {width}] on device {device}, its columns adjacent")
    return stride if n > 1 else w


def _workspace(nbytes, like):
    """A call's own workspace, so that calls on different streams and captured graphs never share one."""
    return _torch.empty(nbytes, dtype=_torch.uint8, device=like.device)


_torch = _int8 = _int32 = _current = None


def _with_torch():
    """torch, imported on the first call that gets tensors, and what every call takes from it."""
    global _torch, _int8, _int32, _current
    import torch

    _int8, _int32 = torch.int8, torch.int32
    _current = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    _torch = torch


def _elsewhere(device, stream, call, *args):
    """The call with the tensors' device and a given stream as the current ones.  Its launches belong there, and so do its
    workspace and new outputs: memory of another stream's may still be in use by that stream's work."""
    _need(device >= 0, "the tensors must be on a GPU")
    _need(stream is None or stream.device_index == device, "the stream must be of the tensors' device")
    with _torch.cuda.device(device), _torch.cuda.stream(stream):
        return call(*args)


def mnmt_pages_fork(pool, table, lens, parent=None, new=None, out=None, stream=None):
    """The next step's tables: row r goes on from row parent[r] (outside the table: empty; None: itself) with room for
    new[r] more tokens.  Returns (table int32 [rows, max_pages], lengths int32 [rows], info int32 [2]: free pages left,
    pages missing); out: these three tensors."""
    if _torch is None:
        _with_torch()
    rows_in, width = table.shape
    rows = rows_in if parent is None else parent.shape[0]
    _, cfg, nbytes = _pool(pool, width, rows)
    at = pool.get_device()
    _ints("table", table, (rows_in, width), at)
    _ints("lens", lens, (rows_in,), at)
    if parent is not None:
        _ints("parent", parent, (rows,), at)
    if new is not None:
        _ints("new", new, (rows,), at)
    if stream is not None or at < 0 or at != _current():
        return _elsewhere(at, stream, mnmt_pages_fork, pool, table, lens, parent, new, out)
    if out is None:
        # one allocation: the lengths and the counts lie behind the table
        flat = _torch.empty(rows * (width + 1) + 2, dtype=_int32, device=pool.device)
        out = (flat[: rows * width].view(rows, width), flat[rows * width: -2], flat[-2:])
    else:
        for name, t, shape in zip(("out[0]", "out[1]", "out[2]"), out, ((rows, width), (rows,), (2,))):
            _ints(name, t, shape, at)
    ws = _workspace(nbytes, pool)
    rc = _lib.mnmt_pages_fork(cfg, pool.data_ptr(), table.data_ptr(), lens.data_ptr(), rows_in, _ptr(parent), _ptr(new),
                              rows, out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(), ws.data_ptr(), nbytes,
                              _stream())
    if rc:
        _check(rc, "mnmt_pages_fork")
    return out


def mnmt_pages_compact(pool, table, lens, out=None, stream=None):
    """Moves the pages in use to the lowest numbers.  Returns (table int32 [rows, max_pages], info int32 [2]: live pages,
    pages moved); out: these two tensors (out[0] may be the table itself)."""
    if _torch is None:
        _with_torch()
    rows, width = table.shape
    _, cfg, nbytes = _pool(pool, width, rows)
    at = pool.get_device()
    _ints("table", table, (rows, width), at)
    _ints("lens", lens, (rows,), at)
    if stream is not None or at < 0 or at != _current():
        return _elsewhere(at, stream, mnmt_pages_compact, pool, table, lens, out)
    if out is None:
        flat = _torch.empty(rows * width + 2, dtype=_int32, device=pool.device)
        out = (flat[:-2].view(rows, width), flat[-2:])
    else:
        _ints("out[0]", out[0], (rows, width), at)
        _ints("out[1]", out[1], (2,), at)
    ws = _workspace(nbytes, pool)
    rc = _lib.mnmt_pages_compact(cfg, pool.data_ptr(), table.data_ptr(), lens.data_ptr(), rows, out[0].data_ptr(),
                                 out[1].data_ptr(), ws.data_ptr(), nbytes, _stream())
    if rc:
        _check(rc, "mnmt_pages_compact")
    return out


def mnmt_pages_write(pool, layer, table, lens, k, v, start=None, max_q=None, stream=None):
    """Writes the codes k, v int8 [n, n_kv_heads * d_head] of new tokens, the last ones of their rows, into a layer's
    pages; row r has the tokens start[r] .. start[r + 1] - 1 (None: n / rows each), at most max_q as far as known."""
    if _torch is None:
        _with_torch()
    rows, width = table.shape
    shape, cfg, _ = _pool(pool, width, rows)
    at = pool.get_device()
    _ints("table", table, (rows, width), at)
    _ints("lens", lens, (rows,), at)
    d = shape.n_kv_heads * shape.d_head
    ld, n = _codes("k", k, d, at), k.shape[0]
    _need(_codes("v", v, d, at) == ld and v.shape[0] == n, "k and v must have the same rows and row stride")
    _need(n < 1 << 31, "there must be fewer than 2^31 tokens")
    if start is not None:
        _ints("start", start, (rows + 1,), at)
    if stream is not None or at < 0 or at != _current():
        return _elsewhere(at, stream, mnmt_pages_write, pool, layer, table, lens, k, v, start, max_q)
    rc = _lib.mnmt_pages_write(cfg, pool.data_ptr(), layer, table.data_ptr(), lens.data_ptr(), rows, k.data_ptr(),
                               v.data_ptr(), ld, _ptr(start), n, n if max_q is None else min(int(max_q), n), _stream())
    if rc:
        _check(rc, "mnmt_pages_write")


def _attn_out(q, kind, out):
    dt = _int8 if kind == ATTN_I8 else _torch.float32
    n, d = q.shape
    if out is None:
        return _torch.empty((n, d), dtype=dt, device=q.device), d
    _need(out.dtype is dt and out.shape == (n, d) and out.device == q.device and (out.numel() == 0 or out.stride(1) == 1),
          f"out must be {dt} [{n}, {d}] on {q.device}, its columns adjacent")
    return out, out.stride(0) if n > 1 else d


def _most(n, rows, start, max_q):
    """The most queries of a row, as far as known."""
    return n // max(rows, 1) if start is None else n if max_q is None or max_q > n else int(max_q)


def mnmt_attn_paged(q, pool, layer, table, lens, c_qk, c_pv, kind=ATTN_F32, start=None, causal=True, max_q=None,
                    max_len=None, out=None, stream=None):
    """Attention of the rows' last tokens, q int8 [n, n_heads * d_head], over a layer's pages: fp32 or (ATTN_I8) int8 of
    q's shape.  Row r has the tokens start[r] .. start[r + 1] - 1 (None: n / rows each); max_q and max_len: the most of
    a row and the longest length, as far as known."""
    if _torch is None:
        _with_torch()
    rows, width = table.shape
    shape, cfg, _ = _pool(pool, width, rows)
    at = pool.get_device()
    _ints("table", table, (rows, width), at)
    _ints("lens", lens, (rows,), at)
    n, d = q.shape
    ld = _codes("q", q, d, at)
    if start is not None:
        _ints("start", start, (rows + 1,), at)
    if stream is not None or at < 0 or at != _current():
        return _elsewhere(at, stream, mnmt_attn_paged, q, pool, layer, table, lens, c_qk, c_pv, kind, start, causal, max_q,
                          max_len, out)
    out, ldo = _attn_out(q, kind, out)
    longest = width * shape.page_size
    a, nbytes = _attn(rows, n, shape.n_kv_heads, shape.d_head, d, kind, 1 if causal else 0, ld, ldo,
                      _most(n, rows, start, max_q), longest if max_len is None else min(int(max_len), longest),
                      float(c_qk), float(c_pv))
    ws = _workspace(nbytes, q) if nbytes else None
    rc = _lib.mnmt_attn_paged(cfg, a, pool.data_ptr(), layer, table.data_ptr(), lens.data_ptr(), rows, q.data_ptr(),
                              _ptr(start), n, out.data_ptr(), _ptr(ws), nbytes, _stream())
    if rc:
        _check(rc, "mnmt_attn_paged")
    return out


def mnmt_attn_cross(q, k, v, lens, d_head, c_qk, c_pv, kind=ATTN_F32, start=None, max_q=None, out=None, stream=None):
    """Attention of q int8 [n, n_heads * d_head] to the keys and values int8 [rows, S, n_kv_heads * d_head] of each
    query's source sentence, lens[b] of them: fp32 or (ATTN_I8) int8 of q's shape.  Sentence b has the queries
    start[b] .. start[b + 1] - 1 (None: n / rows each), at most max_q as far as known."""
    if _torch is None:
        _with_torch()
    rows, S, width = k.shape
    n, d = q.shape
    at = q.get_device()
    _need(d_head > 0 and width > 0 and width % d_head == 0, "k and v must have whole heads")
    batch, ld, one = k.stride()
    if (k.dtype is not _int8 or v.dtype is not _int8 or v.shape != k.shape or k.get_device() != at or v.get_device() != at
            or (rows and S and (one != 1 or v.stride() != k.stride()))):
        raise ValueError(f"k and v must be int8 [rows, S, n_kv_heads * d_head] on {q.device}, strided alike, their columns "
                         "adjacent")
    _ints("lens", lens, (rows,), at)
    ldq = _codes("q", q, d, at)
    if start is not None:
        _ints("start", start, (rows + 1,), at)
    if stream is not None or at < 0 or at != _current():
        return _elsewhere(at, stream, mnmt_attn_cross, q, k, v, lens, d_head, c_qk, c_pv, kind, start, max_q, out)
    out, ldo = _attn_out(q, kind, out)
    hkv = width // d_head
    a, nbytes = _attn(rows, n, hkv, d_head, d, kind, 0, ldq, ldo, _most(n, rows, start, max_q), S, float(c_qk),
                      float(c_pv))
    ws = _workspace(nbytes, q) if nbytes else None
    rc = _lib.mnmt_attn_cross(a, hkv, d_head, k.data_ptr(), v.data_ptr(), ld if S > 1 else width, batch if rows > 1 else 0,
                              S, lens.data_ptr(), rows, q.data_ptr(), _ptr(start), n, out.data_ptr(), _ptr(ws), nbytes,
                              _stream())
    if rc:
        _check(rc, "mnmt_attn_cross")
    return out


class Model:
    """A model loaded into a torch-allocated device arena."""

    def __init__(self, blob: bytes, device="cuda", stream=None, flags: int = 0):
        import torch

        self.arena = torch.empty(mnmt_model_bytes(blob, flags), dtype=torch.uint8, device=device)
        h = C.c_void_p()
        _check(lib().mnmt_model_load_ex(blob, len(blob), flags, _ptr(self.arena), self.arena.numel(),
                                        _stream(stream), C.byref(h)), "mnmt_model_load_ex")
        self.handle = h
        info = ModelInfo()
        _check(lib().mnmt_model_get_info(h, C.byref(info)), "mnmt_model_get_info")
        self.info = info

    def close(self):
        if getattr(self, "handle", None):
            lib().mnmt_model_free(self.handle)
            self.handle = None

    def __del__(self):
        if _lib is not None:
            self.close()


def _settle(t):
    """Wait for the work queued on the current stream of t's device.  The
    allocator may hand out memory that queued kernels still use (it orders
    reuse within that stream only), and mnmt_session_create fills the
    workspace on a stream of its own."""
    import torch

    if t.is_cuda:
        with torch.cuda.device(t.device):  # (memory of a capture is its graph's own)
            if not torch.cuda.is_current_stream_capturing():
                torch.cuda.current_stream(t.device).synchronize()


class Session:
    """Decoding state of one model over a torch-allocated workspace."""

    def __init__(self, model: Model, max_batch: int, max_src_len: int, max_tgt_len: int, beam: int = 1):
        import torch

        self.model = model
        self.cfg = SessionCfg(max_batch, max_src_len, max_tgt_len, beam)
        n = C.c_size_t()
        _check(lib().mnmt_session_bytes(model.handle, C.byref(self.cfg), C.byref(n)), "mnmt_session_bytes")
        self.ws = torch.empty(n.value, dtype=torch.uint8, device=model.arena.device)
        _settle(self.ws)
        h = C.c_void_p()
        _check(lib().mnmt_session_create(model.handle, C.byref(self.cfg), _ptr(self.ws), self.ws.numel(),
                                         C.byref(h)), "mnmt_session_create")
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            lib().mnmt_session_free(self.handle)
            self.handle = None

    def __del__(self):
        if _lib is not None:
            self.close()

    def encode(self, src, lens, stream=None):
        B, S = src.shape
        _check(lib().mnmt_encode(self.handle, _ptr(src), _ptr(lens), B, S, _stream(stream)), "mnmt_encode")
        self._batch = B

    def decode_step(self, prev=None, want_logits=False, stream=None):
        import torch

        B = self._batch
        nxt = torch.empty(B, dtype=torch.int32, device=self.ws.device)
        logits = torch.empty((B, self.model.info.vocab), dtype=torch.float32,
                             device=self.ws.device) if want_logits else None
        _check(lib().mnmt_decode_step(self.handle, _ptr(prev), _ptr(nxt), _ptr(logits), _stream(stream)),
               "mnmt_decode_step")
        return nxt, logits

    def translate(self, src, lens, beam=1, max_steps=None, alpha=0.6, stop_at_eos=False, use_graph=True,
                  stream=None, out=None):
        import torch

        B, S = src.shape
        steps = max_steps or self.cfg.max_tgt_len
        if out is None:
            out = (torch.empty((B, steps), dtype=torch.int32, device=src.device),
                   torch.empty(B, dtype=torch.int32, device=src.device),
                   torch.empty(B, dtype=torch.float32, device=src.device))
        sc = SearchCfg(beam, steps, float(alpha), int(stop_at_eos), int(use_graph))
        _check(lib().mnmt_translate(self.handle, _ptr(src), _ptr(lens), B, S, C.byref(sc), _ptr(out[0]),
                                    _ptr(out[1]), _ptr(out[2]), _stream(stream)), "mnmt_translate")
        return out

    def status(self, stream=None):
        """Synchronize and raise MnmtError(E_TIMEOUT) if a chained kernel's wait gave up."""
        _check(lib().mnmt_session_status(self.handle, _stream(stream)), "mnmt_session_status")

    def tensor(self, name: str, dtype, shape):
        """A view of a session buffer (inside the workspace tensor)."""
        p, n = C.c_void_p(), C.c_size_t()
        _check(lib().mnmt_session_tensor(self.handle, name.encode(), C.byref(p), C.byref(n)), "mnmt_session_tensor")
        off = p.value - self.ws.data_ptr()
        return self.ws[off: off + n.value].view(dtype)[: _numel(shape)].view(shape)


def _numel(shape):
    n = 1
    for s in shape:
        n *= s
    return n
