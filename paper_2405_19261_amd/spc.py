"""Python binding of libspeccascade (the C interface in include/speccascade.h).

Argument marshalling only: every step of the verify path runs in the gfx950
kernels of ``libspeccascade.so``.  Functions carry the C names; tensors are
torch tensors on the current HIP device (PyTorch supplies device memory and
streams, nothing else).  A missing or unloadable library raises -- there is no
fallback implementation.
"""
import ctypes
import os

import torch

# SPC_LIB_PATH selects another build of the library (e.g. a tuning variant)
LIB_PATH = os.environ.get("SPC_LIB_PATH") or os.path.join(
    os.path.dirname(os.path.abspath(__file__)), "libspeccascade.so")

SPC_F32, SPC_BF16, SPC_E4M3 = 0, 1, 2
SPC_RULE_CHOW, SPC_RULE_DIFF, SPC_RULE_OPT, SPC_RULE_ALWAYS, SPC_RULE_NEVER = range(5)
SPC_RULE_TOKEN_V1, SPC_RULE_TOKEN_V2, SPC_RULE_TOKEN_V3 = 5, 6, 7
SPC_RULE_LOSSY, SPC_RULE_BILD, SPC_RULE_CHOWLOG, SPC_RULE_DIFFLOG, SPC_RULE_OPTLOG = range(8, 13)
SPC_MAX_GAMMA = 63
STATUS = {0: "SPC_OK", -1: "SPC_E_NULL", -2: "SPC_E_SHAPE", -3: "SPC_E_RULE",
          -4: "SPC_E_PARAM", -5: "SPC_E_ALIGN", -6: "SPC_E_WORKSPACE", -7: "SPC_E_HIP"}

_P = ctypes.c_void_p
_I32 = ctypes.c_int32


class ExArgs(ctypes.Structure):
    """spc_verify_ex_args."""
    _fields_ = [("rule_per_seq", _P), ("alpha_per_seq", _P), ("temp_per_seq", _P),
                ("out_row_stats", _P), ("out_argmax", _P), ("out_sample_norm", _P),
                ("workspace", _P), ("workspace_bytes", ctypes.c_size_t),
                ("rules_present", ctypes.c_uint32), ("ev_tiles_begin", _P),
                ("ev_tiles_end", _P)]


class Truncation(ctypes.Structure):
    """spc_truncation."""
    _fields_ = [("temperature", ctypes.c_float), ("top_k", _I32), ("top_p", ctypes.c_float),
                ("min_p", ctypes.c_float), ("temp_per_seq", _P), ("top_k_per_seq", _P),
                ("top_p_per_seq", _P), ("min_p_per_seq", _P)]


class KvCache(ctypes.Structure):
    """spc_kv_cache."""
    _fields_ = [("k_pages", _P), ("v_pages", _P), ("k_scale", _P), ("v_scale", _P),
                ("dtype", _I32), ("num_pages", _I32), ("page_size", _I32), ("kv_heads", _I32),
                ("head_dim", _I32), ("page_table", _P), ("table_width", _I32), ("kv_len", _P),
                ("B", _I32)]


class SpcError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


_lib = None


def lib():
    """The loaded shared library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built: run `python -m "
                               "paper_2405_19261_amd.build` (or __graft_entry__.build())")
        L = ctypes.CDLL(LIB_PATH)
        common = [_P, _P, ctypes.c_int]
        L.spc_verify.argtypes = common + [_P, _P, _I32, _I32, _I32, _I32, ctypes.c_float,
                                          ctypes.c_float, _P, _P, _P, _P]
        L.spc_verify.restype = ctypes.c_int
        L.spc_greedy_verify.argtypes = common + [_P, _I32, _I32, _I32, _I32, ctypes.c_float,
                                                 _P, _P, _P, _P]
        L.spc_greedy_verify.restype = ctypes.c_int
        L.spc_verify_ex.argtypes = common + [_P, _P, _I32, _I32, _I32, _I32, ctypes.c_float,
                                             ctypes.c_float, _P, _P, _P,
                                             ctypes.POINTER(ExArgs), _P]
        L.spc_verify_ex.restype = ctypes.c_int
        L.spc_verify_noalloc.argtypes = L.spc_verify_ex.argtypes
        L.spc_verify_noalloc.restype = ctypes.c_int
        L.spc_noalloc_scratch_bytes.argtypes = []
        L.spc_noalloc_scratch_bytes.restype = ctypes.c_size_t
        L.spc_draft_sample.argtypes = [_P, ctypes.c_int, _I32, _I32, ctypes.c_float, _P, _P, _P,
                                       _P]
        L.spc_draft_sample.restype = ctypes.c_int
        L.spc_draft_sample_ws.argtypes = [_P, ctypes.c_int, _I32, _I32, ctypes.c_float, _P, _P,
                                          _P, _P, ctypes.c_size_t, _P]
        L.spc_draft_sample_ws.restype = ctypes.c_int
        L.spc_draft_workspace_bytes.argtypes = [_I32, _I32, ctypes.c_int]
        L.spc_draft_workspace_bytes.restype = ctypes.c_size_t
        cut, cache, i64 = ctypes.POINTER(Truncation), ctypes.POINTER(KvCache), ctypes.c_int64
        L.spc_sample.argtypes = [_P, _I32, _I32, _I32, i64, cut, _P, _P, _P, _P, _P,
                                 ctypes.c_size_t, _P]
        L.spc_sample.restype = ctypes.c_int
        L.spc_truncate.argtypes = [_P, _I32, _I32, _I32, _I32, cut, _P, _P, ctypes.c_size_t, _P]
        L.spc_truncate.restype = ctypes.c_int
        L.spc_truncation_workspace_bytes.argtypes = [i64, _I32, _I32]
        L.spc_truncation_workspace_bytes.restype = ctypes.c_size_t
        L.spc_kv_write.argtypes = [cache, _P, _P, _I32, i64, i64, i64, _P, _P]
        L.spc_kv_write.restype = ctypes.c_int
        L.spc_kv_read.argtypes = [cache, _P, _P, _I32, _I32, _P]
        L.spc_kv_read.restype = ctypes.c_int
        L.spc_kv_attend.argtypes = [cache, _P, _I32, i64, _I32, i64, _P, _I32, ctypes.c_float,
                                    _I32, _P, i64, _P, ctypes.c_size_t, _P]
        L.spc_kv_attend.restype = ctypes.c_int
        L.spc_kv_workspace_bytes.argtypes = [cache, _I32, i64, _I32]
        L.spc_kv_workspace_bytes.restype = ctypes.c_size_t
        L.spc_workspace_bytes.argtypes = [_I32, _I32, _I32, ctypes.c_int]
        L.spc_workspace_bytes.restype = ctypes.c_size_t
        L.spc_workspace_zero_bytes.argtypes = [_I32, _I32, _I32, ctypes.c_int]
        L.spc_workspace_zero_bytes.restype = ctypes.c_size_t
        L.spc_last_error.argtypes = []
        L.spc_last_error.restype = ctypes.c_char_p
        L.spc_release.argtypes = []
        L.spc_release.restype = None
        L.spc_version.argtypes = []
        L.spc_version.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _dtype_code(t):
    if t.dtype == torch.float32:
        return SPC_F32
    if t.dtype == torch.bfloat16:
        return SPC_BF16
    raise TypeError(f"logits must be float32 or bfloat16, not {t.dtype}")


# A call's host side is a few microseconds, as long as the kernel of a small
# step, so it takes addresses as plain integers (the declared argument types
# convert them), names C functions once, and reads the current stream's handle
# without building a Stream object: torch.cuda.current_stream() alone took
# 2.6 us of a 9.1 us call (B = 1, gamma = 4, V = 1000), which takes 6.4 us now.
def _ptr(t):
    return None if t is None else t.data_ptr()


_raw_stream = None  # the current stream's handle, once torch has been asked for a stream


def _stream(stream):
    global _raw_stream
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream()
    handle = torch.cuda.current_stream().cuda_stream  # (initialises torch's HIP state)
    device, current = (getattr(torch._C, n, None)
                       for n in ("_cuda_getDevice", "_cuda_getCurrentRawStream"))
    if device is not None and current is not None:
        _raw_stream = lambda: current(device())  # noqa: E731
    return handle


def _check(status):
    if status != 0:
        raise SpcError(status, lib().spc_last_error().decode())


def _outputs(dev, B, gamma):
    return (torch.empty(B, dtype=torch.int32, device=dev),
            torch.empty(B, dtype=torch.int32, device=dev),
            torch.empty((B, gamma + 1), dtype=torch.uint8, device=dev))


def _shape(q, p, draft):
    qs = q.shape
    if len(qs) != 3 or qs != p.shape or q.dtype != p.dtype:
        raise ValueError("q and p must both be [B, gamma+1, V] of one dtype")
    if not (q.is_contiguous() and p.is_contiguous()):
        raise ValueError("inputs must be contiguous")
    dev = q.device
    if p.device != dev:
        raise ValueError("q and p must be on one device")
    B, g1, V = qs
    _check_arg("draft", draft, torch.int32, dev, (B, g1 - 1))
    return B, g1 - 1, V, dev


def _check_arg(name, t, dtype, device, shape=None):
    """Raise unless t is a contiguous tensor of dtype on device (of shape)."""
    if t is None:
        return
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} must be on {device}, not {t.device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")


# The calls below take many tensors each: one test of everything a tensor must
# be costs less than _check_arg's, one after the other, and _check_arg then
# names what is wrong.  (The binding's share of a cache write: 12.5 us of host
# time with _check_arg alone, 9.3 us with this.)
def _expect(name, t, dtype, like, shape):
    if t is not None and not (t.dtype is dtype and t.get_device() == like.get_device()
                              and t.shape == shape and t.is_contiguous()):
        _check_arg(name, t, dtype, like.device, shape)


def _int32(name, x):
    """x as an integer argument of 32 bits (ctypes alone takes it modulo 2^32)."""
    x = int(x)
    if not -(1 << 31) <= x < 1 << 31:
        raise ValueError(f"{name} must be an integer of 32 bits, not {x}")
    return x


def _on_current_device(t):
    """Raise unless the kernels, which run on the current device, may read t."""
    d = t.get_device()
    if d < 0 or d != torch.cuda.current_device():
        raise ValueError(f"tensors must be on the current HIP device, not {t.device}")


def spc_verify(q, p, draft, uniforms, rule, alpha, temperature, out=None, stream=None):
    """One verify step; returns (accept_len [B], next_token [B], defer_mask [B, gamma+1])."""
    B, gamma, V, dev = _shape(q, p, draft)
    _check_arg("uniforms", uniforms, torch.float32, dev, (B, gamma + 1))
    acc, tok, dm = out if out is not None else _outputs(dev, B, gamma)
    _check(lib().spc_verify(_ptr(q), _ptr(p), _dtype_code(q), _ptr(draft), _ptr(uniforms), B,
                            gamma, V, int(rule), float(alpha), float(temperature), _ptr(acc),
                            _ptr(tok), _ptr(dm), _stream(stream)))
    return acc, tok, dm


def spc_greedy_verify(q, p, draft, rule, alpha, out=None, stream=None):
    """The temperature-0 step; returns (accept_len, next_token, defer_mask)."""
    B, gamma, V, dev = _shape(q, p, draft)
    acc, tok, dm = out if out is not None else _outputs(dev, B, gamma)
    _check(lib().spc_greedy_verify(_ptr(q), _ptr(p), _dtype_code(q), _ptr(draft), B, gamma, V,
                                   int(rule), float(alpha), _ptr(acc), _ptr(tok), _ptr(dm),
                                   _stream(stream)))
    return acc, tok, dm


def _verify_ex(entry, q, p, draft, uniforms, rule, alpha, temperature, rule_per_seq=None,
               alpha_per_seq=None, temp_per_seq=None, out_row_stats=None, out_argmax=None,
               out_sample_norm=None, workspace=None, rules_present=0, ev_tiles=None, out=None,
               stream=None):
    """spc_verify with per-sequence parameters and optional outputs.
    rules_present: bitmask of the rule ids rule_per_seq may hold (0 = any).
    ev_tiles: for profiling, a pair of raw hipEvent_t handles (integers)
    recorded around the statistics kernel of the call's first launch."""
    B, gamma, V, dev = _shape(q, p, draft)
    _check_arg("uniforms", uniforms, torch.float32, dev, (B, gamma + 1))
    _check_arg("rule_per_seq", rule_per_seq, torch.int32, dev, (B,))
    _check_arg("alpha_per_seq", alpha_per_seq, torch.float32, dev, (B,))
    _check_arg("temp_per_seq", temp_per_seq, torch.float32, dev, (B,))
    _check_arg("out_row_stats", out_row_stats, torch.float32, dev, (B, gamma + 1, 8))
    _check_arg("out_argmax", out_argmax, torch.int32, dev, (B, gamma + 1, 2))
    _check_arg("out_sample_norm", out_sample_norm, torch.float32, dev, (B,))
    acc, tok, dm = out if out is not None else _outputs(dev, B, gamma)
    if workspace is not None and (workspace.device != dev or not workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous tensor on the logits' device")
    ex = ExArgs(_ptr(rule_per_seq), _ptr(alpha_per_seq), _ptr(temp_per_seq), _ptr(out_row_stats),
                _ptr(out_argmax), _ptr(out_sample_norm), _ptr(workspace),
                0 if workspace is None else workspace.numel() * workspace.element_size(),
                int(rules_present))
    if ev_tiles is not None:
        ex.ev_tiles_begin, ex.ev_tiles_end = int(ev_tiles[0]), int(ev_tiles[1])
    _check(getattr(lib(), entry)(_ptr(q), _ptr(p), _dtype_code(q), _ptr(draft), _ptr(uniforms), B,
                                  gamma, V, int(rule), float(alpha), float(temperature),
                                  _ptr(acc), _ptr(tok), _ptr(dm), ctypes.byref(ex),
                                  _stream(stream)))
    return acc, tok, dm


def spc_verify_ex(q, p, draft, uniforms, rule, alpha, temperature, **kw):
    """spc_verify with per-sequence parameters and optional outputs (keyword
    arguments of _verify_ex: rule_per_seq, alpha_per_seq, temp_per_seq,
    out_row_stats, out_argmax, out_sample_norm, workspace, rules_present,
    ev_tiles, out, stream); returns (accept_len, next_token, defer_mask)."""
    return _verify_ex("spc_verify_ex", q, p, draft, uniforms, rule, alpha, temperature, **kw)


def spc_verify_noalloc(q, p, draft, uniforms, rule, alpha, temperature, **kw):
    """spc_verify_ex on the library's static scratch: no device allocation
    (``workspace`` must be None)."""
    return _verify_ex("spc_verify_noalloc", q, p, draft, uniforms, rule, alpha, temperature,
                      **kw)


def spc_noalloc_scratch_bytes():
    return lib().spc_noalloc_scratch_bytes()


def spc_draft_sample(logits, temperature, uniforms=None, temp_per_seq=None, out=None,
                     workspace=None, stream=None):
    """The drafter's sampling step: one token per row of ``logits`` [B, V]
    (float32 or bfloat16, contiguous) from softmax(z / T), T = 0 giving the
    argmax.  Returns the tokens [B] int32 (``out`` if given).  ``workspace``:
    an optional caller workspace (a uint8 tensor of at least
    spc_draft_workspace_bytes bytes, zeroed before its first use)."""
    if logits.dim() != 2 or not logits.is_contiguous():
        raise ValueError("logits must be a contiguous [B, V] tensor")
    B, V = logits.shape
    dev = logits.device
    _check_arg("uniforms", uniforms, torch.float32, dev, (B,))
    _check_arg("temp_per_seq", temp_per_seq, torch.float32, dev, (B,))
    tok = out if out is not None else torch.empty(B, dtype=torch.int32, device=dev)
    _check_arg("out", tok, torch.int32, dev, (B,))
    if workspace is None:
        _check(lib().spc_draft_sample(_ptr(logits), _dtype_code(logits), B, V, float(temperature),
                                      _ptr(temp_per_seq), _ptr(uniforms), _ptr(tok),
                                      _stream(stream)))
    else:
        if workspace.device != dev or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor on the logits' device")
        _check(lib().spc_draft_sample_ws(_ptr(logits), _dtype_code(logits), B, V,
                                         float(temperature), _ptr(temp_per_seq), _ptr(uniforms),
                                         _ptr(tok), _ptr(workspace),
                                         workspace.numel() * workspace.element_size(),
                                         _stream(stream)))
    return tok


def _truncation(temperature, top_k, top_p, min_p, temp_per_seq, top_k_per_seq, top_p_per_seq,
                min_p_per_seq, like, B):
    top_k = _int32("top_k", top_k)
    temperature, top_p, min_p = float(temperature), float(top_p), float(min_p)
    if temp_per_seq is top_k_per_seq is top_p_per_seq is min_p_per_seq is None:
        return Truncation(temperature, top_k, top_p, min_p)
    _expect("temp_per_seq", temp_per_seq, torch.float32, like, (B,))
    _expect("top_k_per_seq", top_k_per_seq, torch.int32, like, (B,))
    _expect("top_p_per_seq", top_p_per_seq, torch.float32, like, (B,))
    _expect("min_p_per_seq", min_p_per_seq, torch.float32, like, (B,))
    return Truncation(temperature, top_k, top_p, min_p, _ptr(temp_per_seq),
                      _ptr(top_k_per_seq), _ptr(top_p_per_seq), _ptr(min_p_per_seq))


def _workspace(workspace, like):
    """(address, bytes) of a caller workspace; (None, 0) for the library's own."""
    if workspace is None:
        return None, 0
    if workspace.device != like.device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {like.device}")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def spc_sample(logits, uniforms=None, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, *,
               temp_per_seq=None, top_k_per_seq=None, top_p_per_seq=None, min_p_per_seq=None,
               out=None, out_logprob=None, out_kept=None, workspace=None, stream=None):
    """One token per row of ``logits`` [B, V] (float32 or bfloat16; rows may
    be strided, a row's entries are not) from softmax(z / T) cut by top-k,
    top-p and min-p, at ``uniforms`` [B] (float32).  Returns the tokens [B]
    int32 (``out`` if given; -1 where nothing is kept).  ``out_logprob`` [B]
    float32 and ``out_kept`` [B] int32 receive the token's log-probability
    under the kept distribution and the number of entries kept."""
    if logits.dim() != 2:
        raise ValueError("logits must be a [B, V] tensor")
    B, V = logits.shape
    _int32("the number of rows", B)
    _int32("the length of a row", V)
    if logits.stride(1) != 1 or (B > 1 and logits.stride(0) < V):
        raise ValueError("the entries of a row of logits must be contiguous, rows not overlap")
    _expect("uniforms", uniforms, torch.float32, logits, (B,))
    _expect("out_logprob", out_logprob, torch.float32, logits, (B,))
    _expect("out_kept", out_kept, torch.int32, logits, (B,))
    cut = _truncation(temperature, top_k, top_p, min_p, temp_per_seq, top_k_per_seq,
                      top_p_per_seq, min_p_per_seq, logits, B)
    tok = out if out is not None else torch.empty(B, dtype=torch.int32, device=logits.device)
    _expect("out", tok, torch.int32, logits, (B,))
    code = _dtype_code(logits)
    ws, nbytes = _workspace(workspace, logits)
    _on_current_device(logits)
    _check(lib().spc_sample(_ptr(logits), code, B, V, logits.stride(0) if B > 1 else V, cut,
                            _ptr(uniforms), _ptr(tok), _ptr(out_logprob), _ptr(out_kept), ws,
                            nbytes, _stream(stream)))
    return tok


def spc_truncate(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, *, temp_per_seq=None,
                 top_k_per_seq=None, top_p_per_seq=None, min_p_per_seq=None, out=None,
                 workspace=None, stream=None):
    """``logits`` [B, rows, V] or [B, V] (float32 or bfloat16, contiguous)
    with the entries that top-k, top-p and min-p leave out set to -inf: the
    rows ``spc_verify`` reads when drafts were drawn by ``spc_sample``.
    Returns ``out`` (a new tensor unless given; it may be ``logits``)."""
    if logits.dim() not in (2, 3) or not logits.is_contiguous():
        raise ValueError("logits must be a contiguous [B, rows, V] or [B, V] tensor")
    B, V = logits.shape[0], logits.shape[-1]
    rows = logits.shape[1] if logits.dim() == 3 else 1
    for n in (B, rows, V):
        _int32("a dimension of logits", n)
    cut = _truncation(temperature, top_k, top_p, min_p, temp_per_seq, top_k_per_seq,
                      top_p_per_seq, min_p_per_seq, logits, B)
    if out is None:
        out = torch.empty_like(logits)
    _expect("out", out, logits.dtype, logits, logits.shape)
    code = _dtype_code(logits)
    ws, nbytes = _workspace(workspace, logits)
    _on_current_device(logits)
    _check(lib().spc_truncate(_ptr(logits), code, B, rows, V, cut, _ptr(out), ws, nbytes,
                              _stream(stream)))
    return out


def spc_truncation_workspace_bytes(rows, V, dtype_code):
    return lib().spc_truncation_workspace_bytes(rows, _int32("V", V), dtype_code)


def _kv_cache(k_pages, v_pages, page_table, kv_len, k_scale, v_scale):
    if k_pages.dim() != 4 or v_pages.dim() != 4:
        raise ValueError("k_pages must be [pages, heads, page_size, dim], v_pages "
                         "[pages, heads, dim, page_size]")
    n, H, S, D = k_pages.shape
    dt = k_pages.dtype
    if dt is torch.bfloat16:
        code = SPC_BF16
        if k_scale is not None or v_scale is not None:
            raise ValueError("a bfloat16 cache has no scales")
    elif dt is torch.float8_e4m3fn:
        code = SPC_E4M3
        if k_scale is None or v_scale is None:
            raise ValueError("a float8_e4m3fn cache needs k_scale and v_scale")
        _expect("k_scale", k_scale, torch.float32, k_pages, (n, H, S))
        _expect("v_scale", v_scale, torch.float32, k_pages, (n, H, S))
    else:
        raise TypeError(f"pages must be bfloat16 or float8_e4m3fn, not {dt}")
    if not k_pages.is_contiguous():
        raise ValueError("k_pages must be contiguous")
    _expect("v_pages", v_pages, dt, k_pages, (n, H, D, S))
    if page_table.dim() != 2:
        raise ValueError("page_table must be [B, pages of a sequence]")
    B, width = page_table.shape
    _expect("page_table", page_table, torch.int32, k_pages, (B, width))
    _expect("kv_len", kv_len, torch.int32, k_pages, (B,))
    return KvCache(k_pages.data_ptr(), v_pages.data_ptr(), _ptr(k_scale), _ptr(v_scale), code, n,
                   S, H, D, page_table.data_ptr(), width, kv_len.data_ptr(), B)


def _kv_rows(name, t, like, B, row_start, dim):
    """(rows, heads, stride between rows) of new tokens: [B, n, heads, dim],
    or [rows, heads, dim] with row_start.  Rows may be strided (a slice of a
    fused projection); the heads of a row are contiguous."""
    if row_start is not None:
        _expect("q_start", row_start, torch.int32, like, (B + 1,))
    shape = t.shape
    if len(shape) != (3 if row_start is not None else 4):
        raise ValueError(f"{name} must be [B, n, heads, dim], or [rows, heads, dim] with q_start")
    if t.get_device() != like.get_device():
        raise ValueError(f"{name} must be on {like.device}, not {t.device}")
    heads, d = shape[-2:]
    if d == dim and t.is_contiguous():
        if row_start is not None:
            return shape[0], heads, heads * d
        if shape[0] == B:
            return B * shape[1], heads, heads * d
    if d != dim:
        raise ValueError(f"{name} must have {dim} dimensions a head, not {d}")
    if t.stride(-1) != 1 or (heads > 1 and t.stride(-2) != d):
        raise ValueError(f"the heads of a row of {name} must be contiguous")
    if row_start is not None:
        rows, stride = t.shape[0], t.stride(0)
    else:
        if t.shape[0] != B:
            raise ValueError(f"{name} must hold {B} sequences, not {t.shape[0]}")
        n = t.shape[1]
        rows, stride = B * n, t.stride(1) if n > 1 else t.stride(0)
        if n > 1 and B > 1 and t.stride(0) != n * stride:
            raise ValueError(f"the rows of {name} must be evenly spaced over the batch")
    return rows, heads, heads * d if rows == 1 else stride


def spc_kv_write(k, v, k_pages, v_pages, page_table, kv_len, *, k_scale=None, v_scale=None,
                 q_start=None, stream=None):
    """The keys and values of new tokens (float32 or bfloat16, [B, n, heads,
    dim], or [rows, heads, dim] with ``q_start`` [B + 1]) into the pages of
    their sequences: bfloat16 pages, or float8_e4m3fn with ``k_scale`` and
    ``v_scale``.  The last new token of sequence b is at ``kv_len[b]`` - 1."""
    cache = _kv_cache(k_pages, v_pages, page_table, kv_len, k_scale, v_scale)
    rows, heads, ks = _kv_rows("k", k, k_pages, cache.B, q_start, cache.head_dim)
    vrows, vheads, vs = _kv_rows("v", v, k_pages, cache.B, q_start, cache.head_dim)
    if rows != vrows or not heads == vheads == cache.kv_heads or k.dtype != v.dtype:
        raise ValueError("k and v must have the same rows and type, and the cache's heads")
    code = _dtype_code(k)
    if rows == 0:
        return
    _on_current_device(k_pages)
    _check(lib().spc_kv_write(cache, k.data_ptr(), v.data_ptr(), code, ks, vs, rows,
                              _ptr(q_start), _stream(stream)))


def spc_kv_read(k_pages, v_pages, page_table, kv_len, length=None, *, k_scale=None, v_scale=None,
                dtype=torch.bfloat16, out=None, stream=None):
    """Positions 0 .. ``length`` - 1 of every sequence as dense keys and
    values [B, length, heads, dim] in ``dtype`` (float32 or bfloat16).
    ``out``: a pair to write instead; positions past ``kv_len`` keep what they
    hold (new tensors: zero)."""
    cache = _kv_cache(k_pages, v_pages, page_table, kv_len, k_scale, v_scale)
    if length is not None:
        length = _int32("length", length)
    if out is None:
        if length is None:
            raise ValueError("length or out must be given")
        shape = (cache.B, length, cache.kv_heads, cache.head_dim)
        out = tuple(torch.zeros(shape, dtype=dtype, device=k_pages.device) for _ in range(2))
    k, v = out
    if length is None:
        length = _int32("length", k.shape[1])
    shape = (cache.B, length, cache.kv_heads, cache.head_dim)
    _expect("out", k, k.dtype, k_pages, shape)
    _expect("out", v, k.dtype, k_pages, shape)
    code = _dtype_code(k)
    if length == 0:
        return k, v
    _on_current_device(k_pages)
    _check(lib().spc_kv_read(cache, k.data_ptr(), v.data_ptr(), code, length, _stream(stream)))
    return k, v


def spc_kv_attend(q, k_pages, v_pages, page_table, kv_len, *, scale=None, window=0, k_scale=None,
                  v_scale=None, q_start=None, max_q=None, out=None, workspace=None, stream=None):
    """Attention of new tokens, whose keys and values the cache holds
    already, over the cache: ``q`` bfloat16 [B, n, heads, dim], or [rows,
    heads, dim] with ``q_start`` [B + 1] and ``max_q`` (the most rows of one
    sequence; None: all rows).  ``scale`` None: 1 / sqrt(dim).  ``window`` > 0:
    only the last ``window`` tokens.  Returns ``out`` (as ``q``)."""
    cache = _kv_cache(k_pages, v_pages, page_table, kv_len, k_scale, v_scale)
    dim = cache.head_dim
    rows, heads, qs = _kv_rows("q", q, k_pages, cache.B, q_start, dim)
    if q.dtype is not torch.bfloat16:
        raise TypeError(f"q must be bfloat16, not {q.dtype}")
    if out is None:  # (rows of no sequence stay zero)
        out = (torch.empty if q_start is None else torch.zeros)(q.shape, dtype=q.dtype,
                                                                device=q.device)
    if out.shape != q.shape or out.dtype is not q.dtype:
        raise ValueError("out must have the shape and type of q")
    os_ = _kv_rows("out", out, k_pages, cache.B, q_start, dim)[2]
    ws, nbytes = _workspace(workspace, k_pages)
    window = _int32("window", window)
    most = rows if max_q is None else _int32("max_q", max_q)
    if rows == 0:
        return out
    _on_current_device(k_pages)
    _check(lib().spc_kv_attend(cache, q.data_ptr(), SPC_BF16, qs, heads, rows, _ptr(q_start),
                               most, dim ** -0.5 if scale is None else float(scale), window,
                               out.data_ptr(), os_, ws, nbytes, _stream(stream)))
    return out


def spc_kv_workspace_bytes(k_pages, v_pages, page_table, kv_len, heads, rows, max_q=None, *,
                           k_scale=None, v_scale=None, q_start=None):
    """Bytes of workspace an spc_kv_attend call of this cache and chunk needs:
    ``rows`` rows in all, ``q_start`` and ``max_q`` as the call gets them (with
    ``q_start``, ``max_q`` None: all rows may be one sequence's; a ``max_q`` alone
    stands for a call with ``q_start``)."""
    cache = _kv_cache(k_pages, v_pages, page_table, kv_len, k_scale, v_scale)
    if max_q is None:
        max_q = 0 if q_start is None else rows
    return lib().spc_kv_workspace_bytes(cache, _int32("heads", heads), rows, _int32("max_q", max_q))


def spc_workspace_bytes(B, gamma, V, dtype_code):
    return lib().spc_workspace_bytes(B, gamma, V, dtype_code)


def spc_workspace_zero_bytes(B, gamma, V, dtype_code):
    return lib().spc_workspace_zero_bytes(B, gamma, V, dtype_code)


def spc_draft_workspace_bytes(B, V, dtype_code):
    return lib().spc_draft_workspace_bytes(B, V, dtype_code)


def spc_last_error():
    return lib().spc_last_error().decode()


def spc_release():
    lib().spc_release()


def spc_version():
    return lib().spc_version().decode()
