"""Python binding of the C ABI in include/dspark.h (argument marshalling only).

Every function takes torch tensors that live on a ROCm device, checks their
dtype/shape/contiguity, passes raw pointers to ``libdspark.so`` and raises
``DSparkError`` with the library's message when a call fails.  Outputs that are
not supplied are allocated with torch (device memory plumbing); all
computation happens in the library's HIP kernels, enqueued on the current
torch stream unless ``stream`` is given, whose memory the outputs and workspaces that
a call allocates then are.  There is no fallback: without the built library every
call raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdspark.so")

DSPARK_F32 = 0
DSPARK_BF16 = 1
STATUS = {0: "OK", 1: "EINVAL", 2: "ESHAPE", 3: "EDTYPE", 4: "EUNSUPPORTED", 5: "EWORKSPACE",
          6: "EHIP"}


class DSparkError(RuntimeError):
    def __init__(self, msg: str, status: int = -1):
        super().__init__(msg)
        self.status = status


_lib = None


def lib():
    """The loaded C library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        # DSPARK_LIB: another build of the same library to load instead (the
        # host-sanitizer test builds an instrumented copy)
        path = os.environ.get("DSPARK_LIB") or LIB_PATH
        if not os.path.exists(path):
            raise DSparkError(f"{path} is missing: build it with "
                              "`python -m paper_2607_05147_amd.build` (no fallback path exists)")
        L = C.CDLL(path)
        p, i32, i64, sz, f32 = C.c_void_p, C.c_int, C.c_int64, C.c_size_t, C.c_float
        L.dspark_abi_version.restype = i32
        L.dspark_abi_version.argtypes = []
        L.dspark_last_error.restype = C.c_char_p
        L.dspark_last_error.argtypes = []
        L.dspark_schedule_workspace_size.restype = sz
        L.dspark_schedule_workspace_size.argtypes = [i32, i32]
        L.dspark_schedule.restype = i32
        L.dspark_schedule.argtypes = [p, i32, i32, p, i64, i32, p, p, p, p, sz, p]
        L.dspark_schedule_noalloc.restype = i32
        L.dspark_schedule_noalloc.argtypes = [p, i32, i32, p, i64, i32, p, p, p, p]
        L.dspark_schedule_capacity.restype = i32
        L.dspark_schedule_capacity.argtypes = [p, i32, i32, p, i64, p, p, sz, p]
        L.dspark_schedule_topk.restype = i32
        L.dspark_schedule_topk.argtypes = [p, i32, i32, p, p, p, p, p, sz, p]
        L.dspark_verify_attn_workspace_size.restype = sz
        L.dspark_verify_attn_workspace_size.argtypes = [i32] * 8 + [i32]
        L.dspark_verify_attn.restype = i32
        L.dspark_verify_attn.argtypes = [p, p, p, p, p, p, i32, p, p, i32, i32, i32, i32, i32, i32,
                                         i32, f32, i32, p, p, p, sz, p]
        L.dspark_accept_workspace_size.restype = sz
        L.dspark_accept_workspace_size.argtypes = [i32, i32, i32]
        L.dspark_accept.restype = i32
        L.dspark_accept.argtypes = [p, p, p, i32, i64, p, p, i32, i32, i32, f32, p, p, p, p, sz, p]
        L.dspark_markov_draft_workspace_size.restype = sz
        L.dspark_markov_draft_workspace_size.argtypes = [i32, i32, i32, i32]
        L.dspark_markov_draft.restype = i32
        L.dspark_markov_draft.argtypes = [p, p, i32, i64, p, p, i32, p, p, i32, p, p, f32, i32, i32,
                                          i32, p, p, p, p, sz, p]
        L.dspark_rnn_draft_workspace_size.restype = sz
        L.dspark_rnn_draft_workspace_size.argtypes = [i32, i32, i32, i32]
        L.dspark_rnn_draft.restype = i32
        L.dspark_rnn_draft.argtypes = [p, p, i32, i64, p, p, p, i32, p, p, i32, p, p, f32, i32, i32,
                                       i32, p, p, p, p, sz, p]
        L.dspark_check_verify_inputs.restype = i32
        L.dspark_check_verify_inputs.argtypes = [p, i32, p, p, i32, i32, i32, i32, p, p]
        L.dspark_check_accept_inputs.restype = i32
        L.dspark_check_accept_inputs.argtypes = [p, p, i32, i32, p, p]
        L.dspark_check_schedule_inputs.restype = i32
        L.dspark_check_schedule_inputs.argtypes = [p, i32, i32, p, p]
        L.dspark_check_draft_inputs.restype = i32
        L.dspark_check_draft_inputs.argtypes = [p, p, i32, i32, p, p]
        L.dspark_cache_append.restype = i32
        L.dspark_cache_append.argtypes = [p, p, i64, i64, i32, p, p, p, p, p, p, i32, p, i32, i32, p, p,
                                          i32, i32, i32, i32, i32, i32, p]
        L.dspark_verify_attn_scaled_workspace_size.restype = sz
        L.dspark_verify_attn_scaled_workspace_size.argtypes = [i32] * 10
        L.dspark_verify_attn_scaled.restype = i32
        L.dspark_verify_attn_scaled.argtypes = [p, p, p, p, p, p, p, i32, p, i32, i32, p, p, i32, i32, i32,
                                                i32, i32, i32, i32, f32, i32, p, p, p, sz, p]
        L.dspark_pages_workspace_size.restype = sz
        L.dspark_pages_workspace_size.argtypes = [i32, i32]
        L.dspark_pages_reserve.restype = i32
        L.dspark_pages_reserve.argtypes = [p, i32, p, p, i32, i32, p, i32, p, i32, p, p, sz, p]
        L.dspark_pages_commit.restype = i32
        L.dspark_pages_commit.argtypes = [p, i32, p, p, p, p, i32, i32, p, i32, p]
        L.dspark_pages_trim.restype = i32
        L.dspark_pages_trim.argtypes = [p, i32, p, p, i32, i32, p, i32, p]
        L.dspark_pages_fork.restype = i32
        L.dspark_pages_fork.argtypes = [p, i32, p, i32, i32, p, i32, p, p, p, i32, p, sz, p]
        L.dspark_pages_compact.restype = i32
        L.dspark_pages_compact.argtypes = [p, i32, p, i32, i32, p, i32, p, i32, p, p, sz, p]
        L.dspark_check_page_inputs.restype = i32
        L.dspark_check_page_inputs.argtypes = [p, i32, p, i32, i32, p, i32, p, p]
        _lib = L
    return _lib


def dspark_abi_version() -> int:
    return int(lib().dspark_abi_version())


def dspark_last_error() -> str:
    return lib().dspark_last_error().decode()


def _raise(st: int, what: str) -> None:
    if st != 0:
        raise DSparkError(f"{what}: {STATUS.get(st, st)}: {dspark_last_error()}", st)


def _dev(t: Optional[torch.Tensor], name: str, dtype=None, shape=None, optional=False):
    # (a step's host time is mostly these checks: what passes takes one line)
    if (isinstance(t, torch.Tensor) and t.is_cuda and (dtype is None or t.dtype == dtype) and
            (shape is None or t.shape == shape) and t.is_contiguous()):
        return t
    if t is None:
        if optional:
            return None
        raise DSparkError(f"{name} is required")
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise DSparkError(f"{name} must be a torch tensor on a ROCm device")
    if dtype is not None and t.dtype != dtype:
        raise DSparkError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise DSparkError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise DSparkError(f"{name} must be contiguous")
    return t


def _p(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(stream) -> C.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """What a call allocates is memory of the stream that it runs on: of the current stream's, the
    allocator may give a block that kernels still to come there use, and another stream does not wait
    for them.  The caller may read it on the current stream too, once that waits for the call's."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(torch.cuda.current_stream(t.device))
    return t


def _workspace(nbytes: int, device, ws: Optional[torch.Tensor], stream) -> Tuple[Optional[torch.Tensor], int]:
    if nbytes == 0:
        return ws, 0 if ws is None else ws.numel() * ws.element_size()
    if ws is None:
        ws = _empty(nbytes, torch.uint8, device, stream)
    return ws, ws.numel() * ws.element_size()


_DT = {torch.float32: DSPARK_F32, torch.bfloat16: DSPARK_BF16}


# ------------------------------------------------------------------ stage 1

def dspark_schedule_workspace_size(R: int, K: int) -> int:
    return int(lib().dspark_schedule_workspace_size(R, K))


# ---------------------------------------------------------------- input checks

CHECK_RULES = {
    "verify": {1: "rows of the request outside the batch (or cu_q decreasing)", 2: "q_len above max_q",
               3: "kv_len outside [q_len, max_pages * page_size]", 4: "block-table entry outside the cache"},
    "accept": {1: "rows of the request outside the batch (or cu_q decreasing)", 2: "len = q_len - 1 outside [0, K]",
               3: "uniform outside [0, 1)"},
    "schedule": {1: "confidence outside [0, 1]"},
    "draft": {1: "temperature not finite and positive", 2: "uniform outside [0, 1)"},
    "pages": {1: "kv_len outside [0, max_pages * page_size]", 2: "held table entry outside the cache",
              3: "held table entry names a page without holders",
              4: "held table entry names a page that more entries name than its ref"},
}


def debug_checks() -> bool:
    """DSPARK_DEBUG=1: the stage wrappers check their device-side inputs
    first and raise on the first rule broken (each call then waits for its
    check)."""
    return os.environ.get("DSPARK_DEBUG", "0") not in ("", "0")


def _report(report: torch.Tensor, kind: str, stream) -> Optional[tuple]:
    (torch.cuda.current_stream(report.device) if stream is None else stream).synchronize()
    code, r, i, v = (int(x) for x in report.cpu().tolist())
    return None if code == 0 else (code, r, i, v, CHECK_RULES[kind].get(code, "?"))


def check_verify_inputs(block_table: torch.Tensor, kv_len: torch.Tensor, cu_q: torch.Tensor, max_q: int,
                        page_size: int, num_pages: int, stream=None) -> Optional[tuple]:
    """First broken rule of dspark_verify_attn's device-side inputs as
    (code, request, index, value, rule) or None; waits for the check."""
    _dev(block_table, "block_table", torch.int32)
    R, max_pages = block_table.shape
    _dev(kv_len, "kv_len", torch.int32, (R,))
    _dev(cu_q, "cu_q", torch.int32, (R + 1,))
    report = _empty(4, torch.int32, cu_q.device, stream)
    st = lib().dspark_check_verify_inputs(_p(block_table), max_pages, _p(kv_len), _p(cu_q), R, max_q,
                                          page_size, num_pages, _p(report), _stream(stream))
    _raise(st, "dspark_check_verify_inputs")
    return _report(report, "verify", stream)


def check_accept_inputs(cu_q: torch.Tensor, u: Optional[torch.Tensor], K: int, stream=None) -> Optional[tuple]:
    _dev(cu_q, "cu_q", torch.int32)
    R = cu_q.numel() - 1
    _dev(u, "u", torch.float32, (R, K + 1), optional=True)
    report = _empty(4, torch.int32, cu_q.device, stream)
    st = lib().dspark_check_accept_inputs(_p(cu_q), _p(u), R, K, _p(report), _stream(stream))
    _raise(st, "dspark_check_accept_inputs")
    return _report(report, "accept", stream)


def check_schedule_inputs(conf: torch.Tensor, stream=None) -> Optional[tuple]:
    _dev(conf, "conf", torch.float32)
    R, K = conf.shape
    report = _empty(4, torch.int32, conf.device, stream)
    st = lib().dspark_check_schedule_inputs(_p(conf), R, K, _p(report), _stream(stream))
    _raise(st, "dspark_check_schedule_inputs")
    return _report(report, "schedule", stream)


def check_draft_inputs(u: torch.Tensor, sts_temp: Optional[torch.Tensor] = None,
                       stream=None) -> Optional[tuple]:
    """First broken rule of a draft block's uniforms [R, K] and per-position
    temperatures [K] (request -1) as (code, request, index, value, rule) or
    None; waits for the check."""
    _dev(u, "u", torch.float32)
    R, K = u.shape
    _dev(sts_temp, "sts_temp", torch.float32, (K,), optional=True)
    report = _empty(4, torch.int32, u.device, stream)
    st = lib().dspark_check_draft_inputs(_p(u), _p(sts_temp), R, K, _p(report), _stream(stream))
    _raise(st, "dspark_check_draft_inputs")
    return _report(report, "draft", stream)


def check_page_inputs(block_table: torch.Tensor, kv_len: torch.Tensor, page_size: int, ref: torch.Tensor,
                      stream=None) -> Optional[tuple]:
    """First broken rule of the dspark_pages_* state as (code, request, index,
    value, rule) or None; waits for the check."""
    R, max_pages, num_pages = _page_state(block_table, kv_len, ref)
    report = _empty(4, torch.int32, ref.device, stream)
    st = lib().dspark_check_page_inputs(_p(block_table), max_pages, _p(kv_len), R, page_size, _p(ref), num_pages,
                                        _p(report), _stream(stream))
    _raise(st, "dspark_check_page_inputs")
    return _report(report, "pages", stream)


def _cache_pages(cache: torch.Tensor, strides: Sequence[int], heads: int, page_size: int, dim: int) -> int:
    """Pages a flat cache holds: page p is readable when its last element,
    p * s0 + (heads - 1) * s1 + (page_size - 1) * s2 + dim - 1, is inside."""
    s0, s1, s2 = strides
    s0, s1, s2 = int(s0), int(s1), int(s2)
    span = (heads - 1) * s1 + (page_size - 1) * s2 + dim
    return max(0, (cache.numel() - span) // s0 + 1) if s0 > 0 else 0


def _debug_raise(found: Optional[tuple], what: str) -> None:
    if found is not None:
        code, r, i, v, rule = found
        raise DSparkError(f"{what}: input check failed: request {r}: {rule} (code {code}, index {i}, "
                          f"value {v})", 1)


def dspark_schedule(conf: torch.Tensor, sps: torch.Tensor, mode: int = 0,
                    len_out: Optional[torch.Tensor] = None, cu_q: Optional[torch.Tensor] = None,
                    tok_req: Optional[torch.Tensor] = None, want_tok_req: bool = False,
                    ws: Optional[torch.Tensor] = None, stream=None):
    """conf fp32 [R, K], sps fp64 [> R*(K+1)] -> (len int32 [R], cu_q int32 [R+1], tok_req|None)."""
    _dev(conf, "conf", torch.float32)
    if conf.dim() != 2:
        raise DSparkError("conf must be [R, K]")
    R, K = conf.shape
    _dev(sps, "sps", torch.float64)
    dev = conf.device
    if len_out is None:
        len_out = _empty(R, torch.int32, dev, stream)
    if cu_q is None:
        cu_q = _empty(R + 1, torch.int32, dev, stream)
    if tok_req is None and want_tok_req:
        tok_req = _empty(R * (K + 1), torch.int32, dev, stream)
    _dev(len_out, "len", torch.int32, (R,))
    _dev(cu_q, "cu_q", torch.int32, (R + 1,))
    _dev(tok_req, "tok_req", torch.int32, (R * (K + 1),), optional=True)
    ws, ws_bytes = _workspace(dspark_schedule_workspace_size(R, K), dev, ws, stream)
    if debug_checks() and K > 0:
        _debug_raise(check_schedule_inputs(conf, stream), "dspark_schedule")
    st = lib().dspark_schedule(_p(conf), R, K, _p(sps), sps.numel(), mode, _p(len_out), _p(cu_q),
                               _p(tok_req), _p(ws), ws_bytes, _stream(stream))
    _raise(st, "dspark_schedule")
    return len_out, cu_q, tok_req


def dspark_schedule_noalloc(conf: torch.Tensor, sps: torch.Tensor, mode: int,
                            len_out: torch.Tensor, cu_q: torch.Tensor,
                            tok_req: Optional[torch.Tensor] = None, stream=None):
    """As dspark_schedule, with the library's fixed scratch array as workspace;
    every output is the caller's (nothing is allocated)."""
    _dev(conf, "conf", torch.float32)
    if conf.dim() != 2:
        raise DSparkError("conf must be [R, K]")
    R, K = conf.shape
    _dev(sps, "sps", torch.float64)
    _dev(len_out, "len", torch.int32, (R,))
    _dev(cu_q, "cu_q", torch.int32, (R + 1,))
    _dev(tok_req, "tok_req", torch.int32, (R * (K + 1),), optional=True)
    st = lib().dspark_schedule_noalloc(_p(conf), R, K, _p(sps), sps.numel(), mode, _p(len_out),
                                       _p(cu_q), _p(tok_req), _stream(stream))
    _raise(st, "dspark_schedule_noalloc")
    return len_out, cu_q, tok_req


def dspark_schedule_capacity(conf_prev: torch.Tensor, sps: torch.Tensor,
                             capacity: Optional[torch.Tensor] = None,
                             ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """conf_prev fp32 [R, K], sps fp64 [> R*(K+1)] -> capacity int32 [1] (device)."""
    _dev(conf_prev, "conf_prev", torch.float32)
    if conf_prev.dim() != 2:
        raise DSparkError("conf_prev must be [R, K]")
    R, K = conf_prev.shape
    _dev(sps, "sps", torch.float64)
    dev = conf_prev.device
    if capacity is None:
        capacity = _empty(1, torch.int32, dev, stream)
    _dev(capacity, "capacity", torch.int32, (1,))
    ws, ws_bytes = _workspace(dspark_schedule_workspace_size(R, K), dev, ws, stream)
    st = lib().dspark_schedule_capacity(_p(conf_prev), R, K, _p(sps), sps.numel(), _p(capacity),
                                        _p(ws), ws_bytes, _stream(stream))
    _raise(st, "dspark_schedule_capacity")
    return capacity


def dspark_schedule_topk(conf: torch.Tensor, capacity: torch.Tensor,
                         len_out: Optional[torch.Tensor] = None,
                         cu_q: Optional[torch.Tensor] = None,
                         tok_req: Optional[torch.Tensor] = None, want_tok_req: bool = False,
                         ws: Optional[torch.Tensor] = None, stream=None):
    """conf fp32 [R, K], capacity int32 [1] (device) -> (len, cu_q, tok_req|None)."""
    _dev(conf, "conf", torch.float32)
    if conf.dim() != 2:
        raise DSparkError("conf must be [R, K]")
    R, K = conf.shape
    _dev(capacity, "capacity", torch.int32, (1,))
    dev = conf.device
    if len_out is None:
        len_out = _empty(R, torch.int32, dev, stream)
    if cu_q is None:
        cu_q = _empty(R + 1, torch.int32, dev, stream)
    if tok_req is None and want_tok_req:
        tok_req = _empty(R * (K + 1), torch.int32, dev, stream)
    _dev(len_out, "len", torch.int32, (R,))
    _dev(cu_q, "cu_q", torch.int32, (R + 1,))
    _dev(tok_req, "tok_req", torch.int32, (R * (K + 1),), optional=True)
    ws, ws_bytes = _workspace(dspark_schedule_workspace_size(R, K), dev, ws, stream)
    st = lib().dspark_schedule_topk(_p(conf), R, K, _p(capacity), _p(len_out), _p(cu_q),
                                    _p(tok_req), _p(ws), ws_bytes, _stream(stream))
    _raise(st, "dspark_schedule_topk")
    return len_out, cu_q, tok_req


# ------------------------------------------------------------------ stage 2

def dspark_verify_attn_workspace_size(R: int, max_q: int, Hq: int, Hkv: int, Dqk: int, Dv: int,
                                      max_pages: int, page_size: int, dtype: torch.dtype) -> int:
    return int(lib().dspark_verify_attn_workspace_size(R, max_q, Hq, Hkv, Dqk, Dv, max_pages,
                                                       page_size, _DT[dtype]))


def dspark_verify_attn(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                       k_strides: Sequence[int], v_strides: Sequence[int],
                       block_table: torch.Tensor, kv_len: torch.Tensor, cu_q: torch.Tensor,
                       max_q: int, Hkv: int, Dv: int, page_size: int, scale: float,
                       out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                       want_lse: bool = False, ws: Optional[torch.Tensor] = None, stream=None):
    """q [total_q(or more rows), Hq, Dqk]; caches flat or shaped, addressed by element strides.
    Returns (out [rows of q, Hq, Dv], lse|None)."""
    if q.dtype not in _DT:
        raise DSparkError("q must be float32 or bfloat16")
    _dev(q, "q")
    if q.dim() != 3:
        raise DSparkError("q must be [tokens, Hq, Dqk]")
    rows, Hq, Dqk = q.shape
    _dev(k_cache, "k_cache", q.dtype)
    _dev(v_cache, "v_cache", q.dtype)
    _dev(block_table, "block_table", torch.int32)
    if block_table.dim() != 2:
        raise DSparkError("block_table must be [R, max_pages]")
    R, max_pages = block_table.shape
    _dev(kv_len, "kv_len", torch.int32, (R,))
    _dev(cu_q, "cu_q", torch.int32, (R + 1,))
    if out is None:
        out = _empty((rows, Hq, Dv), q.dtype, q.device, stream)
    _dev(out, "out", q.dtype, (rows, Hq, Dv))
    if lse is None and want_lse:
        lse = _empty((rows, Hq), torch.float32, q.device, stream)
    _dev(lse, "lse", torch.float32, (rows, Hq), optional=True)
    need = dspark_verify_attn_workspace_size(R, max_q, Hq, Hkv, Dqk, Dv, max_pages, page_size,
                                             q.dtype)
    ws, ws_bytes = _workspace(need, q.device, ws, stream)
    if debug_checks():
        num_pages = min(_cache_pages(k_cache, k_strides, Hkv, page_size, Dqk),
                        _cache_pages(v_cache, v_strides, Hkv, page_size, Dv))
        _debug_raise(check_verify_inputs(block_table, kv_len, cu_q, max_q, page_size, max(num_pages, 1),
                                         stream), "dspark_verify_attn")
    ks = (C.c_int64 * 3)(*[int(x) for x in k_strides])
    vs = (C.c_int64 * 3)(*[int(x) for x in v_strides])
    st = lib().dspark_verify_attn(_p(q), _p(k_cache), _p(v_cache), ks, vs, _p(block_table),
                                  max_pages, _p(kv_len), _p(cu_q), R, max_q, Hq, Hkv, Dqk, Dv,
                                  page_size, float(scale), _DT[q.dtype], _p(out), _p(lse), _p(ws),
                                  ws_bytes, _stream(stream))
    _raise(st, "dspark_verify_attn")
    return out, lse


# ------------------------------------------------------------------ the cache in 8 bits

_CODES = (torch.uint8, torch.float8_e4m3fn)


def _on(stream, *tensors) -> int:
    """The stream's handle; every tensor has to be on its device, the current one."""
    here = torch.cuda.current_device()
    if stream is not None and stream.device.index != here:
        raise DSparkError(f"the call's stream is on {stream.device}, the current device is {here}")
    for t in tensors:
        if t is not None and (not isinstance(t, torch.Tensor) or t.get_device() != here):
            raise DSparkError(f"a tensor on {getattr(t, 'device', None)}, the call's stream on device {here}")
    # (the handle alone: an object for the current stream takes longer than a launch)
    return torch._C._cuda_getCurrentRawStream(here) if stream is None else stream.cuda_stream


def _scaled_cache(k_cache, v_cache, k_strides, v_strides, k_scale, v_scale, block, block_table, kv_len, cu_q, page_size,
                  Dqk, Dv):
    """Checks of a cache of e4m3 codes; returns (R, max_pages, num_pages, Hkv)."""
    if block < 1 or page_size < 1 or page_size % block:
        raise DSparkError(f"block={block} must divide page_size={page_size}")
    _dev(k_scale, "k_scale", torch.float32)
    if k_scale.dim() != 3 or k_scale.shape[2] != page_size // block:
        raise DSparkError("k_scale must be [num_pages, Hkv, page_size / block]")
    num_pages, Hkv = k_scale.shape[:2]
    for t, st, sc, D, name in ((k_cache, k_strides, k_scale, Dqk, "k"), (v_cache, v_strides, v_scale, Dv, "v")):
        if t is None:
            continue
        _dev(t, name + "_cache")
        if t.dtype not in _CODES:
            raise DSparkError(f"{name}_cache must be uint8 or float8_e4m3fn, got {t.dtype}")
        _dev(sc, name + "_scale", torch.float32, k_scale.shape)
        if _cache_pages(t, st, Hkv, page_size, D) < num_pages:
            raise DSparkError(f"{name}_cache holds fewer than {num_pages} pages of these strides")
    _dev(block_table, "block_table", torch.int32)
    if block_table.dim() != 2:
        raise DSparkError("block_table must be [R, max_pages]")
    R, max_pages = block_table.shape
    _dev(kv_len, "kv_len", torch.int32, (R,))
    _dev(cu_q, "cu_q", torch.int32, (R + 1,))
    return R, max_pages, num_pages, Hkv


_Strides3 = C.c_int64 * 3


def _strides3(st):
    return _Strides3(*map(int, st))


def _new_rows(t, name, dtype, Hkv):
    """[rows, Hkv, D] whose rows may lie apart: (D, row stride)."""
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda" or t.dim() != 3 or t.dtype != dtype:
        raise DSparkError(f"{name} must be a [rows, Hkv, D] {dtype} ROCm tensor")
    D = t.shape[2]
    if t.shape[1] != Hkv or (D > 1 and t.stride(2) != 1) or (Hkv > 1 and t.stride(1) != D):
        raise DSparkError(f"{name} must have Hkv={Hkv} heads, dense within a row")
    return D, t.stride(0) if t.shape[0] > 1 else max(t.stride(0), Hkv * D)


def dspark_cache_append(k: torch.Tensor, v: Optional[torch.Tensor], k_cache: torch.Tensor,
                        v_cache: Optional[torch.Tensor], k_strides: Sequence[int],
                        v_strides: Optional[Sequence[int]], k_scale: torch.Tensor,
                        v_scale: Optional[torch.Tensor], block: int, block_table: torch.Tensor,
                        kv_len: torch.Tensor, cu_q: torch.Tensor, max_q: int, page_size: int, stream=None) -> None:
    """k [rows, Hkv, Dqk], v [rows, Hkv, Dv] (fp32/bf16, rows may be a part of wider ones) ->
    codes in k_cache, v_cache (uint8 or float8_e4m3fn, flat or shaped, addressed by strides in bytes)
    and fp32 k_scale, v_scale [num_pages, Hkv, page_size / block], in place.  v, v_cache and v_scale
    None: keys alone."""
    if not isinstance(k, torch.Tensor) or k.dtype not in _DT:
        raise DSparkError("k must be float32 or bfloat16")
    if (v is None) != (v_cache is None) or (v is None) != (v_scale is None) or (v is not None and v_strides is None):
        raise DSparkError("v, v_cache, v_strides and v_scale go together")
    Hkv = k.shape[1] if k.dim() == 3 else 0
    Dqk, k_ld = _new_rows(k, "k", k.dtype, Hkv)
    Dv, v_ld = (0, 0) if v is None else _new_rows(v, "v", k.dtype, Hkv)
    if v is not None and v.shape[0] != k.shape[0]:
        raise DSparkError("k and v must have the same rows")
    R, max_pages, num_pages, heads = _scaled_cache(k_cache, v_cache, k_strides, v_strides, k_scale, v_scale, block,
                                                   block_table, kv_len, cu_q, page_size, Dqk, Dv)
    if heads != Hkv:
        raise DSparkError(f"k has {Hkv} heads, k_scale {heads}")
    on = _on(stream, k, v, k_cache, v_cache, k_scale, v_scale, block_table, kv_len, cu_q)
    if debug_checks():
        _debug_raise(check_verify_inputs(block_table, kv_len, cu_q, max_q, page_size, num_pages, stream),
                     "dspark_cache_append")
    st = lib().dspark_cache_append(_p(k), _p(v), k_ld, v_ld,
                                   _DT[k.dtype], _p(k_cache), _p(v_cache), _strides3(k_strides),
                                   None if v is None else _strides3(v_strides), _p(k_scale), _p(v_scale), block,
                                   _p(block_table), max_pages, num_pages, _p(kv_len), _p(cu_q), R, max_q, Hkv, Dqk, Dv,
                                   page_size, on)
    _raise(st, "dspark_cache_append")


def dspark_verify_attn_scaled_workspace_size(R: int, max_q: int, Hq: int, Hkv: int, Dqk: int, Dv: int, max_pages: int,
                                             page_size: int, block: int, dtype: torch.dtype) -> int:
    return int(lib().dspark_verify_attn_scaled_workspace_size(R, max_q, Hq, Hkv, Dqk, Dv, max_pages, page_size, block,
                                                              _DT[dtype]))


def dspark_verify_attn_scaled(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                              k_strides: Sequence[int], v_strides: Sequence[int], k_scale: torch.Tensor,
                              v_scale: torch.Tensor, block: int, block_table: torch.Tensor, kv_len: torch.Tensor,
                              cu_q: torch.Tensor, max_q: int, Dv: int, page_size: int, scale: float,
                              out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                              want_lse: bool = False, ws: Optional[torch.Tensor] = None, stream=None):
    """dspark_verify_attn over a cache of e4m3 codes and scales (dspark_cache_append's).
    q [total_q(or more rows), Hq, Dqk]; returns (out [rows of q, Hq, Dv], lse|None)."""
    _dev(q, "q")
    if q.dtype not in _DT or q.dim() != 3:
        raise DSparkError("q must be a float32 or bfloat16 [tokens, Hq, Dqk] tensor")
    rows, Hq, Dqk = q.shape
    R, max_pages, num_pages, Hkv = _scaled_cache(k_cache, v_cache, k_strides, v_strides, k_scale, v_scale, block,
                                                 block_table, kv_len, cu_q, page_size, Dqk, Dv)
    if out is None:
        out = _empty((rows, Hq, Dv), q.dtype, q.device, stream)
    _dev(out, "out", q.dtype, (rows, Hq, Dv))
    if lse is None and want_lse:
        lse = _empty((rows, Hq), torch.float32, q.device, stream)
    _dev(lse, "lse", torch.float32, (rows, Hq), optional=True)
    if ws is None:
        need = dspark_verify_attn_scaled_workspace_size(R, max_q, Hq, Hkv, Dqk, Dv, max_pages, page_size, block, q.dtype)
        ws, ws_bytes = _workspace(need, q.device, None, stream)
    else:
        ws_bytes = ws.numel() * ws.element_size()
    on = _on(stream, q, k_cache, v_cache, k_scale, v_scale, block_table, kv_len, cu_q, out, lse, ws)
    if debug_checks():
        _debug_raise(check_verify_inputs(block_table, kv_len, cu_q, max_q, page_size, num_pages, stream),
                     "dspark_verify_attn_scaled")
    st = lib().dspark_verify_attn_scaled(_p(q), _p(k_cache), _p(v_cache), _strides3(k_strides), _strides3(v_strides),
                                         _p(k_scale), _p(v_scale), block, _p(block_table), max_pages, num_pages,
                                         _p(kv_len), _p(cu_q), R, max_q, Hq, Hkv, Dqk, Dv, page_size, float(scale),
                                         _DT[q.dtype], _p(out), _p(lse), _p(ws), ws_bytes, on)
    _raise(st, "dspark_verify_attn_scaled")
    return out, lse


# ------------------------------------------------------------------ the pages of a cache

class _PageBuffer(C.Structure):
    _fields_ = [("base", C.c_void_p), ("page_stride", C.c_int64), ("page_bytes", C.c_int64)]


class PageBuffers:
    """The memory that a cache's pages are made of: contiguous tensors of num_pages equal parts
    (keys, values and scales, layer by layer).  Keeps the tensors alive; made once for a cache."""

    def __init__(self, tensors: Sequence[torch.Tensor], num_pages: int):
        self.tensors, self.num_pages = list(tensors), num_pages
        self.array = (_PageBuffer * max(1, len(self.tensors)))()
        for i, t in enumerate(self.tensors):
            _dev(t, f"buffer {i}")
            if t.device != self.tensors[0].device:
                raise DSparkError("the buffers of a cache are on one device")
            n = t.numel() * t.element_size()
            if num_pages < 1 or n == 0 or n % num_pages:
                raise DSparkError(f"buffer {i}: {n} bytes are not {num_pages} pages")
            self.array[i] = _PageBuffer(t.data_ptr(), n // num_pages, n // num_pages)


def page_buffers(tensors: Sequence[torch.Tensor], num_pages: int) -> PageBuffers:
    return PageBuffers(tensors, num_pages)


def dspark_pages_workspace_size(R: int, num_pages: int) -> int:
    return int(lib().dspark_pages_workspace_size(R, num_pages))


def _page_state(block_table, kv_len, ref):
    _dev(block_table, "block_table", torch.int32)
    if block_table.dim() != 2:
        raise DSparkError("block_table must be [R, max_pages]")
    R, max_pages = block_table.shape
    _dev(kv_len, "kv_len", torch.int32, (R,))
    _dev(ref, "ref", torch.int32)
    if ref.dim() != 1:
        raise DSparkError("ref must be [num_pages]")
    return R, max_pages, ref.shape[0]


def _page_call(block_table, kv_len, page_size, ref, bufs, ws, what, stream, *more):
    """What reserve, fork and compact share: sizes, buffers, workspace, the stream and the state's check."""
    R, max_pages, num_pages = _page_state(block_table, kv_len, ref)
    if bufs is not None and bufs.num_pages != num_pages:
        raise DSparkError(f"bufs hold {bufs.num_pages} pages, ref {num_pages}")
    if ws is None:
        ws, ws_bytes = _workspace(dspark_pages_workspace_size(R, num_pages), ref.device, None, stream)
    else:
        ws_bytes = ws.numel() * ws.element_size()
    on = _on(stream, block_table, kv_len, ref, ws, *more, *([] if bufs is None else bufs.tensors[:1]))
    if debug_checks():
        _debug_raise(check_page_inputs(block_table, kv_len, page_size, ref, stream), what)
    return R, max_pages, num_pages, ws, ws_bytes, on


def dspark_pages_reserve(block_table: torch.Tensor, kv_len: torch.Tensor, cu_q: torch.Tensor, page_size: int,
                         ref: torch.Tensor, bufs: Optional[PageBuffers] = None, step_len: Optional[torch.Tensor] = None,
                         ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Pages for cu_q[r+1] - cu_q[r] more tokens of each request; block_table and ref change in place.
    Returns step_len int32 [R], the kv_len of the step (0: not served).  bufs: what is copied where a
    partly filled page is shared (None: nothing)."""
    R, max_pages, num_pages, ws, ws_bytes, on = _page_call(block_table, kv_len, page_size, ref, bufs, ws,
                                                           "dspark_pages_reserve", stream, cu_q, step_len)
    _dev(cu_q, "cu_q", torch.int32, (R + 1,))
    if step_len is None:
        step_len = _empty(R, torch.int32, ref.device, stream)
    _dev(step_len, "step_len", torch.int32, (R,))
    st = lib().dspark_pages_reserve(_p(block_table), max_pages, _p(kv_len), _p(cu_q), R, page_size, _p(ref), num_pages,
                                    None if bufs is None else bufs.array, 0 if bufs is None else len(bufs.tensors),
                                    _p(step_len), _p(ws), ws_bytes, on)
    _raise(st, "dspark_pages_reserve")
    return step_len


def dspark_pages_commit(block_table: torch.Tensor, kv_len: torch.Tensor, step_len: torch.Tensor, cu_q: torch.Tensor,
                        page_size: int, ref: torch.Tensor, accepted_len: Optional[torch.Tensor] = None,
                        stream=None) -> None:
    """After a step: each request keeps 1 + accepted_len of its tokens (None: all); kv_len and ref change in place."""
    R, max_pages, num_pages = _page_state(block_table, kv_len, ref)
    _dev(step_len, "step_len", torch.int32, (R,))
    _dev(cu_q, "cu_q", torch.int32, (R + 1,))
    _dev(accepted_len, "accepted_len", torch.int32, (R,), optional=True)
    on = _on(stream, block_table, kv_len, step_len, cu_q, accepted_len, ref)
    if debug_checks():  # (of the lengths that the step has, whose pages are given back)
        _debug_raise(check_page_inputs(block_table, step_len, page_size, ref, stream), "dspark_pages_commit")
    st = lib().dspark_pages_commit(_p(block_table), max_pages, _p(kv_len), _p(step_len), _p(cu_q), _p(accepted_len), R,
                                   page_size, _p(ref), num_pages, on)
    _raise(st, "dspark_pages_commit")


def dspark_pages_trim(block_table: torch.Tensor, kv_len: torch.Tensor, new_len: torch.Tensor, page_size: int,
                      ref: torch.Tensor, stream=None) -> None:
    """kv_len = min(kv_len, new_len) (0: the request ends); kv_len and ref change in place."""
    R, max_pages, num_pages = _page_state(block_table, kv_len, ref)
    _dev(new_len, "new_len", torch.int32, (R,))
    on = _on(stream, block_table, kv_len, new_len, ref)
    if debug_checks():
        _debug_raise(check_page_inputs(block_table, kv_len, page_size, ref, stream), "dspark_pages_trim")
    st = lib().dspark_pages_trim(_p(block_table), max_pages, _p(kv_len), _p(new_len), R, page_size, _p(ref), num_pages,
                                 on)
    _raise(st, "dspark_pages_trim")


def dspark_pages_fork(block_table: torch.Tensor, kv_len: torch.Tensor, page_size: int, ref: torch.Tensor,
                      parent: torch.Tensor, child: torch.Tensor, len: Optional[torch.Tensor] = None,
                      ws: Optional[torch.Tensor] = None, stream=None) -> None:
    """Requests child [n] (of length 0) share the pages of parent [n], up to len [n] tokens (None: all);
    block_table, kv_len and ref change in place."""
    R, max_pages, num_pages, ws, ws_bytes, on = _page_call(block_table, kv_len, page_size, ref, None, ws,
                                                           "dspark_pages_fork", stream, parent, child, len)
    _dev(parent, "parent", torch.int32)
    n = parent.numel()
    _dev(parent, "parent", torch.int32, (n,))
    _dev(child, "child", torch.int32, (n,))
    _dev(len, "len", torch.int32, (n,), optional=True)
    st = lib().dspark_pages_fork(_p(block_table), max_pages, _p(kv_len), R, page_size, _p(ref), num_pages, _p(parent),
                                 _p(child), _p(len), n, _p(ws), ws_bytes, on)
    _raise(st, "dspark_pages_fork")


def dspark_pages_compact(block_table: torch.Tensor, kv_len: torch.Tensor, page_size: int, ref: torch.Tensor,
                         bufs: Optional[PageBuffers] = None, used: Optional[torch.Tensor] = None,
                         ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Moves the pages in use to ids 0 .. used - 1; block_table, ref and the buffers change in place.
    Returns used int32 [1] (device)."""
    R, max_pages, num_pages, ws, ws_bytes, on = _page_call(block_table, kv_len, page_size, ref, bufs, ws,
                                                           "dspark_pages_compact", stream, used)
    if used is None:
        used = _empty(1, torch.int32, ref.device, stream)
    _dev(used, "used", torch.int32, (1,))
    st = lib().dspark_pages_compact(_p(block_table), max_pages, _p(kv_len), R, page_size, _p(ref), num_pages,
                                    None if bufs is None else bufs.array, 0 if bufs is None else len(bufs.tensors),
                                    _p(used), _p(ws), ws_bytes, on)
    _raise(st, "dspark_pages_compact")
    return used


# ------------------------------------------------------------------ stage 3

def dspark_accept_workspace_size(R: int, K: int, V: int) -> int:
    return int(lib().dspark_accept_workspace_size(R, K, V))


def dspark_accept(draft_tok: torch.Tensor, logits: torch.Tensor, cu_q: torch.Tensor,
                  draft_p: Optional[torch.Tensor] = None, u: Optional[torch.Tensor] = None,
                  inv_temperature: float = 1.0, accepted_len: Optional[torch.Tensor] = None,
                  next_tok: Optional[torch.Tensor] = None, accept_rate: Optional[torch.Tensor] = None,
                  want_rate: bool = False, ws: Optional[torch.Tensor] = None, stream=None):
    """draft_tok int32 [R, K]; logits [rows, V] (fp32/bf16, row stride = stride(0));
    draft_p fp32 [R, K, V] and u fp32 [R, K+1] for stochastic acceptance (both None: greedy).
    Returns (accepted_len int32 [R], next_tok int32 [R], accept_rate|None)."""
    _dev(draft_tok, "draft_tok", torch.int32)
    if draft_tok.dim() != 2:
        raise DSparkError("draft_tok must be [R, K]")
    R, K = draft_tok.shape
    if logits.dtype not in _DT or logits.dim() != 2 or logits.device.type != "cuda":
        raise DSparkError("logits must be a 2-D float32/bfloat16 ROCm tensor")
    if logits.stride(1) != 1:
        raise DSparkError("logits rows must be contiguous")
    V = logits.shape[1]
    ld = logits.stride(0)
    _dev(cu_q, "cu_q", torch.int32, (R + 1,))
    _dev(draft_p, "draft_p", torch.float32, (R, K, V), optional=True)
    _dev(u, "u", torch.float32, (R, K + 1), optional=True)
    dev = draft_tok.device
    if accepted_len is None:
        accepted_len = _empty(R, torch.int32, dev, stream)
    if next_tok is None:
        next_tok = _empty(R, torch.int32, dev, stream)
    if accept_rate is None and want_rate:
        accept_rate = _empty(R * (K + 1), torch.float32, dev, stream)
    _dev(accepted_len, "accepted_len", torch.int32, (R,))
    _dev(next_tok, "next_tok", torch.int32, (R,))
    _dev(accept_rate, "accept_rate", torch.float32, optional=True)
    need = dspark_accept_workspace_size(R, K, V)
    ws, ws_bytes = _workspace(need, dev, ws, stream)
    if debug_checks():
        _debug_raise(check_accept_inputs(cu_q, u, K, stream), "dspark_accept")
    st = lib().dspark_accept(_p(draft_tok), _p(draft_p), C.c_void_p(logits.data_ptr()),
                             _DT[logits.dtype], ld, _p(u), _p(cu_q), R, K, V,
                             float(inv_temperature), _p(accepted_len), _p(next_tok),
                             _p(accept_rate), _p(ws), ws_bytes, _stream(stream))
    _raise(st, "dspark_accept")
    return accepted_len, next_tok, accept_rate


def dspark_markov_draft_workspace_size(R: int, K: int, V: int, rank: int) -> int:
    return int(lib().dspark_markov_draft_workspace_size(R, K, V, rank))


def dspark_markov_draft(anchor: torch.Tensor, base_logits: torch.Tensor, W1: torch.Tensor,
                        W2t: torch.Tensor, w_conf: torch.Tensor, u: torch.Tensor, K: int,
                        hidden: Optional[torch.Tensor] = None,
                        sts_temp: Optional[torch.Tensor] = None, inv_temperature: float = 1.0,
                        draft_tok: Optional[torch.Tensor] = None,
                        draft_p: Optional[torch.Tensor] = None, conf: Optional[torch.Tensor] = None,
                        ws: Optional[torch.Tensor] = None, stream=None):
    """anchor int32 [R]; base_logits [R*K, V] (fp32/bf16, row stride = stride(0));
    W1, W2t bf16 [V, rank]; w_conf fp32 [d + rank]; u fp32 [R, K]; hidden bf16
    [R, K, d] or None; sts_temp fp32 [K] or None.
    Returns (draft_tok int32 [R, K], draft_p fp32 [R, K, V], conf fp32 [R, K])."""
    _dev(anchor, "anchor", torch.int32)
    R = anchor.shape[0]
    if base_logits.dtype not in _DT or base_logits.dim() != 2 or base_logits.device.type != "cuda":
        raise DSparkError("base_logits must be a 2-D float32/bfloat16 ROCm tensor")
    if base_logits.stride(1) != 1 or base_logits.shape[0] != R * K:
        raise DSparkError("base_logits must be [R*K, V] with contiguous rows")
    V = base_logits.shape[1]
    ld = base_logits.stride(0)
    _dev(W1, "W1", torch.bfloat16)
    rank = W1.shape[1]
    _dev(W2t, "W2t", torch.bfloat16, (V, rank))
    if W1.shape != (V, rank):
        raise DSparkError("W1 must be [V, rank]")
    d = 0 if hidden is None else hidden.shape[-1]
    _dev(hidden, "hidden", torch.bfloat16, (R, K, d), optional=True)
    _dev(w_conf, "w_conf", torch.float32, (d + rank,))
    _dev(sts_temp, "sts_temp", torch.float32, (K,), optional=True)
    _dev(u, "u", torch.float32, (R, K))
    dev = anchor.device
    if draft_tok is None:
        draft_tok = _empty((R, K), torch.int32, dev, stream)
    if draft_p is None:
        draft_p = _empty((R, K, V), torch.float32, dev, stream)
    if conf is None:
        conf = _empty((R, K), torch.float32, dev, stream)
    _dev(draft_tok, "draft_tok", torch.int32, (R, K))
    _dev(draft_p, "draft_p", torch.float32, (R, K, V))
    _dev(conf, "conf", torch.float32, (R, K))
    need = dspark_markov_draft_workspace_size(R, K, V, rank)
    if need == 0:
        raise DSparkError(f"unsupported shape: R={R} V={V} rank={rank}")
    ws, ws_bytes = _workspace(need, dev, ws, stream)
    if debug_checks():
        _debug_raise(check_draft_inputs(u, sts_temp, stream), "dspark_markov_draft")
    st = lib().dspark_markov_draft(_p(anchor), C.c_void_p(base_logits.data_ptr()),
                                   _DT[base_logits.dtype], ld, _p(W1), _p(W2t), rank, _p(hidden),
                                   _p(w_conf), d, _p(sts_temp), _p(u), float(inv_temperature), R,
                                   K, V, _p(draft_tok), _p(draft_p), _p(conf), _p(ws), ws_bytes,
                                   _stream(stream))
    _raise(st, "dspark_markov_draft")
    return draft_tok, draft_p, conf


def dspark_rnn_draft_workspace_size(R: int, K: int, V: int, rank: int) -> int:
    return int(lib().dspark_rnn_draft_workspace_size(R, K, V, rank))


def dspark_rnn_draft(anchor: torch.Tensor, base_logits: torch.Tensor, W1: torch.Tensor,
                     W2t: torch.Tensor, Wrnn: torch.Tensor, w_conf: torch.Tensor, u: torch.Tensor,
                     K: int, hidden: Optional[torch.Tensor] = None,
                     sts_temp: Optional[torch.Tensor] = None, inv_temperature: float = 1.0,
                     draft_tok: Optional[torch.Tensor] = None,
                     draft_p: Optional[torch.Tensor] = None, conf: Optional[torch.Tensor] = None,
                     ws: Optional[torch.Tensor] = None, stream=None):
    """As dspark_markov_draft, plus Wrnn bf16 [3 rank, 2 rank + d] (gate,
    candidate and output rows; columns [s; e; h]).
    Returns (draft_tok int32 [R, K], draft_p fp32 [R, K, V], conf fp32 [R, K])."""
    _dev(anchor, "anchor", torch.int32)
    R = anchor.shape[0]
    if base_logits.dtype not in _DT or base_logits.dim() != 2 or base_logits.device.type != "cuda":
        raise DSparkError("base_logits must be a 2-D float32/bfloat16 ROCm tensor")
    if base_logits.stride(1) != 1 or base_logits.shape[0] != R * K:
        raise DSparkError("base_logits must be [R*K, V] with contiguous rows")
    V = base_logits.shape[1]
    ld = base_logits.stride(0)
    _dev(W1, "W1", torch.bfloat16)
    rank = W1.shape[1]
    _dev(W2t, "W2t", torch.bfloat16, (V, rank))
    if W1.shape != (V, rank):
        raise DSparkError("W1 must be [V, rank]")
    d = 0 if hidden is None else hidden.shape[-1]
    _dev(hidden, "hidden", torch.bfloat16, (R, K, d), optional=True)
    _dev(Wrnn, "Wrnn", torch.bfloat16, (3 * rank, 2 * rank + d))
    _dev(w_conf, "w_conf", torch.float32, (d + rank,))
    _dev(sts_temp, "sts_temp", torch.float32, (K,), optional=True)
    _dev(u, "u", torch.float32, (R, K))
    dev = anchor.device
    if draft_tok is None:
        draft_tok = _empty((R, K), torch.int32, dev, stream)
    if draft_p is None:
        draft_p = _empty((R, K, V), torch.float32, dev, stream)
    if conf is None:
        conf = _empty((R, K), torch.float32, dev, stream)
    _dev(draft_tok, "draft_tok", torch.int32, (R, K))
    _dev(draft_p, "draft_p", torch.float32, (R, K, V))
    _dev(conf, "conf", torch.float32, (R, K))
    need = dspark_rnn_draft_workspace_size(R, K, V, rank)
    if need == 0:
        raise DSparkError(f"unsupported shape: R={R} V={V} rank={rank}")
    ws, ws_bytes = _workspace(need, dev, ws, stream)
    if debug_checks():
        _debug_raise(check_draft_inputs(u, sts_temp, stream), "dspark_rnn_draft")
    st = lib().dspark_rnn_draft(_p(anchor), C.c_void_p(base_logits.data_ptr()),
                                _DT[base_logits.dtype], ld, _p(W1), _p(W2t), _p(Wrnn), rank,
                                _p(hidden), _p(w_conf), d, _p(sts_temp), _p(u),
                                float(inv_temperature), R, K, V, _p(draft_tok), _p(draft_p),
                                _p(conf), _p(ws), ws_bytes, _stream(stream))
    _raise(st, "dspark_rnn_draft")
    return draft_tok, draft_p, conf
