"""ctypes binding to libvatp.so: the same four calls as include/vatp.h, taking torch tensors.

Argument marshalling only - every step of the path runs in the CUDA kernels of the library.
There is no fallback: if the library is missing the import raises.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

# VATP_LIBRARY selects another build of the library (the bounds-checking build libvatp_dbg.so)
_LIB_PATH = os.environ.get("VATP_LIBRARY") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "libvatp.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2406_12335_b200.build`")
lib = C.CDLL(_LIB_PATH)

OK = 0
BF16, F32 = 0, 1
IND_H2O, IND_WINDOW = 0, 1
NORM_KINDS = {"l1": 0, "l2": 1, "linf": 2}
FLAG_DECODE_OVERLAP = 1
STATIC_SCRATCH_BYTES = (4 << 20) + 256
EXPORTS = ["vatp_cache_capacity", "vatp_workspace_bytes", "vatp_prefill_scores", "vatp_prefill_scores_from_lse", "vatp_prefill_attention_scores", "vatp_prefill_scores_static", "vatp_select", "vatp_compact", "vatp_compact_window", "vatp_decode_step",
           "vatp_compact_q4", "vatp_cache_pack_q4", "vatp_cache_unpack_q4", "vatp_decode_step_q4", "vatp_cache_copy", "vatp_cache_copy_q4",
           "vatp_selftest_bounded_wait", "vatp_selftest_overlap_policy", "vatp_status_string"]


class Params(C.Structure):
    _fields_ = [("batch", C.c_int32), ("heads", C.c_int32), ("seq_len", C.c_int32), ("head_dim", C.c_int32),
                ("dtype", C.c_int32), ("indicator", C.c_int32), ("window_w", C.c_int32), ("scale", C.c_float),
                ("budget", C.c_int32), ("n_sink", C.c_int32), ("n_recent", C.c_int32), ("norm_kind", C.c_int32),
                ("flags", C.c_int32), ("kv_heads", C.c_int32), ("stride_b", C.c_int64), ("stride_h", C.c_int64), ("stride_t", C.c_int64)]


class CacheStruct(C.Structure):
    _fields_ = [("k_cache", C.c_void_p), ("v_cache", C.c_void_p), ("acc", C.c_void_p), ("vnorm", C.c_void_p),
                ("pos", C.c_void_p), ("len", C.c_void_p), ("free_slot", C.c_void_p), ("next_pos", C.c_void_p),
                ("ring", C.c_void_p), ("acc_fixed", C.c_void_p), ("last_slot", C.c_void_p)]


class CacheQ4Struct(C.Structure):
    _fields_ = [("state", CacheStruct), ("k_params", C.c_void_p), ("v_params", C.c_void_p)]


SEQ_FREE, SEQ_KEEP = -1, -2        # entries of vatp_cache_copy's map that name no source

_vp = C.c_void_p
lib.vatp_cache_capacity.restype = C.c_int32
lib.vatp_cache_capacity.argtypes = [C.c_int32]
lib.vatp_workspace_bytes.restype = C.c_size_t
lib.vatp_workspace_bytes.argtypes = [C.POINTER(Params)]
lib.vatp_prefill_scores.restype = C.c_int
lib.vatp_prefill_scores.argtypes = [C.POINTER(Params), _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, C.c_size_t, _vp, _vp]
lib.vatp_prefill_scores_from_lse.restype = C.c_int
lib.vatp_prefill_scores_from_lse.argtypes = [C.POINTER(Params), _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, C.c_size_t, _vp, _vp]
lib.vatp_prefill_attention_scores.restype = C.c_int
lib.vatp_prefill_attention_scores.argtypes = [C.POINTER(Params), _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, C.c_size_t, _vp, _vp]
lib.vatp_prefill_scores_static.restype = C.c_int
lib.vatp_prefill_scores_static.argtypes = [C.POINTER(Params), _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
lib.vatp_select.restype = C.c_int
lib.vatp_select.argtypes = [C.POINTER(Params), _vp, _vp, _vp, C.c_size_t, _vp, _vp]
lib.vatp_compact.restype = C.c_int
lib.vatp_compact.argtypes = [C.POINTER(Params), _vp, _vp, _vp, _vp, _vp, _vp, C.POINTER(CacheStruct), _vp, _vp]
lib.vatp_compact_window.restype = C.c_int
lib.vatp_compact_window.argtypes = [C.POINTER(Params), _vp, _vp, _vp, _vp, _vp, _vp, _vp, C.POINTER(CacheStruct), _vp, _vp]
lib.vatp_decode_step.restype = C.c_int
lib.vatp_decode_step.argtypes = [C.POINTER(Params), C.POINTER(CacheStruct), _vp, _vp, _vp, _vp, _vp, _vp, _vp]
lib.vatp_compact_q4.restype = C.c_int
lib.vatp_compact_q4.argtypes = [C.POINTER(Params), _vp, _vp, _vp, _vp, _vp, _vp, C.POINTER(CacheQ4Struct), _vp, _vp]
lib.vatp_cache_pack_q4.restype = C.c_int
lib.vatp_cache_pack_q4.argtypes = [C.POINTER(Params), C.POINTER(CacheStruct), C.POINTER(CacheQ4Struct), _vp, _vp]
lib.vatp_cache_unpack_q4.restype = C.c_int
lib.vatp_cache_unpack_q4.argtypes = [C.POINTER(Params), C.POINTER(CacheQ4Struct), C.POINTER(CacheStruct), _vp, _vp]
lib.vatp_decode_step_q4.restype = C.c_int
lib.vatp_decode_step_q4.argtypes = [C.POINTER(Params), C.POINTER(CacheQ4Struct), _vp, _vp, _vp, _vp, _vp, _vp, _vp]
lib.vatp_cache_copy.restype = C.c_int
lib.vatp_cache_copy.argtypes = [C.POINTER(Params), C.POINTER(CacheStruct), C.c_int32, C.c_int32, C.POINTER(CacheStruct), _vp, _vp, _vp]
lib.vatp_cache_copy_q4.restype = C.c_int
lib.vatp_cache_copy_q4.argtypes = [C.POINTER(Params), C.POINTER(CacheQ4Struct), C.c_int32, C.c_int32, C.POINTER(CacheQ4Struct), _vp, _vp, _vp]
lib.vatp_selftest_bounded_wait.restype = C.c_int
lib.vatp_selftest_bounded_wait.argtypes = [C.c_uint64, _vp, _vp, _vp]
lib.vatp_selftest_overlap_policy.restype = C.c_int32
lib.vatp_selftest_overlap_policy.argtypes = [_vp, C.POINTER(C.c_uint64), C.POINTER(C.c_uint64), C.c_int32, C.c_double]
lib.vatp_status_string.restype = C.c_char_p
lib.vatp_status_string.argtypes = [C.c_int]


class VatpError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {lib.vatp_status_string(code).decode()} ({code})")


def _check(code: int, where: str):
    if code != OK:
        raise VatpError(code, where)


def _ptr(t):
    return None if t is None else t.data_ptr()


# current_stream() builds a Stream object, 3.3 us of an 8.5 us call; this asks for the handle alone, 0.3 us.  It is not part
# of torch's public interface: a torch without it takes the longer way.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    return torch.cuda.current_stream().cuda_stream if _raw_stream is None else _raw_stream(torch.cuda.current_device())


def make_params(*, batch, heads, seq_len, head_dim, dtype, budget, n_sink=0, n_recent=0, scale=None,
                indicator="h2o", window=0, strides=(0, 0, 0), norm="l1", decode_overlap=False, kv_heads=0) -> Params:
    """norm: the value norm of Eq. 4, "l1" (the method) or the Ablation Study's "l2" / "linf".
    decode_overlap: sets VATP_FLAG_DECODE_OVERLAP (decode steps of independent caches may run side by side;
    see vatp_decode_step in include/vatp.h for what the caller then guarantees)."""
    dt = {torch.bfloat16: BF16, torch.float32: F32, "bf16": BF16, "f32": F32}[dtype]
    return Params(batch, heads, seq_len, head_dim, dt, IND_WINDOW if indicator == "window" else IND_H2O, window,
                  float(scale if scale is not None else head_dim ** -0.5), budget, n_sink, n_recent, NORM_KINDS[norm],
                  FLAG_DECODE_OVERLAP if decode_overlap else 0, kv_heads, *strides)


def params_for(x: torch.Tensor, **kw) -> Params:
    """Params for a [batch, heads, T, d] tensor, taking shape, dtype and strides from it."""
    b, h, T, d = x.shape
    assert x.stride(3) == 1
    return make_params(batch=b, heads=h, seq_len=T, head_dim=d, dtype=x.dtype,
                       strides=(x.stride(0), x.stride(1), x.stride(2)), **kw)


def vatp_workspace_bytes(p: Params) -> int:
    return int(lib.vatp_workspace_bytes(C.byref(p)))


def _shape(p: Params):
    """What the arrays of a decode state depend on, its batch and budget first and the type of 16- and 32-bit rows last."""
    return p.batch, p.budget, p.kv_heads or p.heads, p.head_dim, p.window_w if p.indicator == IND_WINDOW else 0, p.dtype


class _State:
    """The per-slot and per-unit arrays that both forms of the decode state have."""

    def __init__(self, p: Params, device, share):
        b, h, cap = p.batch, (p.kv_heads or p.heads), int(lib.vatp_cache_capacity(p.budget))
        self.cap, self.budget, self.batch = cap, p.budget, b
        self.made_for = _shape(p)
        if share is not None:
            if (share.cap, share.budget, share.pos.shape[:2]) != (cap, p.budget, (b, h)) or (share.ring is not None) != (p.indicator == IND_WINDOW) \
                    or (share.ring is not None and share.ring.shape[2] != p.window_w):
                raise ValueError("share: a state of other parameters")
            for name in ("acc", "vnorm", "pos", "len", "free_slot", "next_pos", "last_slot", "ring", "acc_fixed"):
                setattr(self, name, getattr(share, name))
            return
        self.acc = torch.zeros(b, h, cap, dtype=torch.float32, device=device)
        self.vnorm = torch.zeros(b, h, cap, dtype=torch.float32, device=device)
        self.pos = torch.full((b, h, cap), -1, dtype=torch.int32, device=device)
        self.len = torch.zeros(b, h, dtype=torch.int32, device=device)
        self.free_slot = torch.zeros(b, h, dtype=torch.int32, device=device)
        self.next_pos = torch.zeros(b, h, dtype=torch.int32, device=device)
        self.last_slot = torch.full((b, h), -1, dtype=torch.int32, device=device)
        self.ring = self.acc_fixed = None
        if p.indicator == IND_WINDOW:
            self.ring = torch.zeros(b, h, p.window_w, cap, dtype=torch.float32, device=device)
            self.acc_fixed = torch.zeros(b, h, cap, dtype=torch.int64, device=device)

    def _struct(self, k, v):
        return CacheStruct(*[_ptr(t) for t in (k, v, self.acc, self.vnorm, self.pos, self.len, self.free_slot, self.next_pos, self.ring,
                                               self.acc_fixed, self.last_slot)])


class Cache(_State):
    """Device arrays of the decode state (allocated with torch, owned by this object).  share: a state of the same parameters
    (the 4-bit form of the same rows) whose arrays other than the rows this one uses too."""

    def __init__(self, p: Params, device="cuda", share=None):
        super().__init__(p, device, share)
        b, h, d = p.batch, (p.kv_heads or p.heads), p.head_dim
        dt = torch.float32 if p.dtype == F32 else torch.bfloat16
        self.k_cache = torch.zeros(b, h, self.cap, d, dtype=dt, device=device)
        self.v_cache = torch.zeros(b, h, self.cap, d, dtype=dt, device=device)
        self.struct = self._struct(self.k_cache, self.v_cache)

    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in (self.k_cache, self.v_cache, self.acc, self.vnorm, self.pos))


class CacheQ4(_State):
    """The decode state with K and V rows in 4 bits (vatp_cache_q4 in include/vatp.h has the format): codes [.., cap, head_dim / 2] uint8
    and params [.., cap, head_dim / 32, 2] bf16 (scale, low end).  share: as for Cache."""

    def __init__(self, p: Params, device="cuda", share=None):
        super().__init__(p, device, share)
        b, h, d = p.batch, (p.kv_heads or p.heads), p.head_dim
        for name in ("k", "v"):
            setattr(self, name + "_codes", torch.zeros(b, h, self.cap, d // 2, dtype=torch.uint8, device=device))
            setattr(self, name + "_params", torch.zeros(b, h, self.cap, d // 32, 2, dtype=torch.bfloat16, device=device))
        self.struct = CacheQ4Struct(self._struct(self.k_codes, self.v_codes), _ptr(self.k_params), _ptr(self.v_params))

    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in (self.k_codes, self.v_codes, self.k_params, self.v_params, self.acc, self.vnorm, self.pos))


def vatp_prefill_scores(p: Params, q, k, v, *, lse_out=None, attn_acc, vnorm, score, win_rows=None,
                        workspace=None, dev_status=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib.vatp_prefill_scores(C.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(lse_out), _ptr(attn_acc), _ptr(vnorm),
                                   _ptr(score), _ptr(win_rows), _ptr(workspace), ws_bytes, _ptr(dev_status),
                                   _stream(stream)), "vatp_prefill_scores")


def vatp_prefill_scores_from_lse(p: Params, q, k, v, lse_in, *, lse_out=None, attn_acc, vnorm, score, win_rows=None,
                                 workspace=None, dev_status=None, stream=None):
    """vatp_prefill_scores with the row normalisers (natural-log lse of the causal softmax rows, as an
    attention forward returns them) given: pass 1 is skipped, QK^T is recomputed once."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib.vatp_prefill_scores_from_lse(C.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(lse_in), _ptr(lse_out),
                                            _ptr(attn_acc), _ptr(vnorm), _ptr(score), _ptr(win_rows), _ptr(workspace),
                                            ws_bytes, _ptr(dev_status), _stream(stream)), "vatp_prefill_scores_from_lse")


def vatp_prefill_attention_scores(p: Params, q, k, v, attn_out, *, lse_out=None, attn_acc, vnorm, score, win_rows=None,
                                  workspace=None, dev_status=None, stream=None):
    """Attention forward fused with prefill scoring: also writes the layer's output rows attn_out
    [batch, heads, T, head_dim] (Eq. 1); the indicator then costs one recomputation of QK^T."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib.vatp_prefill_attention_scores(C.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(attn_out), _ptr(lse_out),
                                             _ptr(attn_acc), _ptr(vnorm), _ptr(score), _ptr(win_rows), _ptr(workspace),
                                             ws_bytes, _ptr(dev_status), _stream(stream)), "vatp_prefill_attention_scores")


def vatp_prefill_scores_static(p: Params, q, k, v, *, lse_out=None, attn_acc, vnorm, score, win_rows=None,
                               dev_status=None, stream=None):
    """vatp_prefill_scores without a workspace argument: for callers that cannot allocate device
    memory, the scratch is a fixed array inside the library (at most STATIC_SCRATCH_BYTES of row
    normalisers; larger problems raise VatpError).  All calls on a device share that array, so
    calls that could overlap on the GPU must be serialised by the caller."""
    _check(lib.vatp_prefill_scores_static(C.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(lse_out), _ptr(attn_acc),
                                          _ptr(vnorm), _ptr(score), _ptr(win_rows), _ptr(dev_status),
                                          _stream(stream)), "vatp_prefill_scores_static")


def vatp_select(p: Params, score, kept_idx, *, workspace=None, dev_status=None, stream=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib.vatp_select(C.byref(p), _ptr(score), _ptr(kept_idx), _ptr(workspace), ws_bytes, _ptr(dev_status),
                           _stream(stream)), "vatp_select")


def vatp_compact(p: Params, k, v, attn_acc, vnorm, kept_idx, cache: Cache, *, win_rows=None, dev_status=None,
                 stream=None):
    _check(lib.vatp_compact(C.byref(p), _ptr(k), _ptr(v), _ptr(attn_acc), _ptr(vnorm), _ptr(win_rows), _ptr(kept_idx),
                            C.byref(cache.struct), _ptr(dev_status), _stream(stream)), "vatp_compact")


def vatp_compact_window(p: Params, q, k, v, lse, attn_acc, vnorm, kept_idx, cache: Cache, *, dev_status=None, stream=None):
    """vatp_compact for the history-window indicator without win_rows: the kept block of the last-w
    probability rows is recomputed from q, the compacted keys and the row normalisers `lse` (natural log)."""
    _check(lib.vatp_compact_window(C.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(lse), _ptr(attn_acc), _ptr(vnorm),
                                   _ptr(kept_idx), C.byref(cache.struct), _ptr(dev_status), _stream(stream)),
           "vatp_compact_window")


def vatp_decode_step(p: Params, cache: Cache, q_new, k_new, v_new, out, *, evicted_pos=None, dev_status=None,
                     stream=None):
    _check(lib.vatp_decode_step(C.byref(p), C.byref(cache.struct), _ptr(q_new), _ptr(k_new), _ptr(v_new), _ptr(out),
                                _ptr(evicted_pos), _ptr(dev_status), _stream(stream)), "vatp_decode_step")


def vatp_compact_q4(p: Params, k, v, attn_acc, vnorm, kept_idx, cache: CacheQ4, *, win_rows=None, dev_status=None, stream=None):
    """vatp_compact into the 4-bit state."""
    _check(lib.vatp_compact_q4(C.byref(p), _ptr(k), _ptr(v), _ptr(attn_acc), _ptr(vnorm), _ptr(win_rows), _ptr(kept_idx),
                               C.byref(cache.struct), _ptr(dev_status), _stream(stream)), "vatp_compact_q4")


def vatp_cache_pack_q4(p: Params, src: Cache, dst: CacheQ4, *, dev_status=None, stream=None):
    """A decode state into one with 4-bit rows; arrays that both share stay as they are."""
    _check(lib.vatp_cache_pack_q4(C.byref(p), C.byref(src.struct), C.byref(dst.struct), _ptr(dev_status), _stream(stream)),
           "vatp_cache_pack_q4")


def vatp_cache_unpack_q4(p: Params, src: CacheQ4, dst: Cache, *, dev_status=None, stream=None):
    """The reverse: rows become the values that their codes stand for, rounded to the params dtype."""
    _check(lib.vatp_cache_unpack_q4(C.byref(p), C.byref(src.struct), C.byref(dst.struct), _ptr(dev_status), _stream(stream)),
           "vatp_cache_unpack_q4")


def vatp_decode_step_q4(p: Params, cache: CacheQ4, q_new, k_new, v_new, out, *, evicted_pos=None, dev_status=None, stream=None):
    """vatp_decode_step on the 4-bit state."""
    _check(lib.vatp_decode_step_q4(C.byref(p), C.byref(cache.struct), _ptr(q_new), _ptr(k_new), _ptr(v_new), _ptr(out),
                                   _ptr(evicted_pos), _ptr(dev_status), _stream(stream)), "vatp_decode_step_q4")


def vatp_cache_copy(p: Params, src, dst, src_of, *, dev_status=None, stream=None):
    """Entry b of `dst` (which p describes) becomes entry src_of[b] of `src`; SEQ_KEEP leaves it, SEQ_FREE empties it.  src_of: int32
    [p.batch] on the device; both states Cache (vatp_cache_copy) or both CacheQ4 (vatp_cache_copy_q4).  A map of another type, length
    or device and states that do not fit p or one another are a ValueError."""
    if type(src) is not type(dst):
        raise TypeError("both states must hold their rows in the same form")
    n = -1 if isinstance(dst, CacheQ4) else None                   # (4-bit rows: whatever type they came from)
    if dst.made_for[:n] != _shape(p)[:n] or src.made_for[2:n] != dst.made_for[2:n]:
        raise ValueError("a state of other parameters")
    if src_of is not None and (src_of.dtype != torch.int32 or src_of.shape != (p.batch,) or not src_of.is_contiguous() or src_of.device != dst.pos.device):
        raise ValueError("src_of: int32, one for each entry of dst, contiguous, where dst is")
    name = "vatp_cache_copy_q4" if isinstance(dst, CacheQ4) else "vatp_cache_copy"
    _check(getattr(lib, name)(C.byref(p), C.byref(src.struct), src.batch, src.budget, C.byref(dst.struct), _ptr(src_of), _ptr(dev_status),
                              _stream(stream)), name)


def vatp_selftest_bounded_wait(limit_ns: int, dev_status, waited_ns=None, *, stream=None):
    """Launches the one-CTA kernel that waits `limit_ns` on a barrier nobody arms and then reports
    VATP_ERR_TIMEOUT (5) in dev_status: shows that an expired device-side wait ends cleanly."""
    _check(lib.vatp_selftest_bounded_wait(int(limit_ns), _ptr(dev_status), _ptr(waited_ns), _stream(stream)),
           "vatp_selftest_bounded_wait")
