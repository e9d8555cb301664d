"""Binding of ``include/bcast_serve.h``: same names, torch tensors in place of pointers.

The extension module (``csrc/serve_bind.cpp``) checks that the tensors have the shapes and types of one
call, describes them to the C entry point of the same name (which checks ranges, alignment and strides) and
returns what it writes; nothing is computed in Python.  Tensors are taken with their strides and are never
copied; the innermost dimension has to be contiguous.  The ``*Args`` classes are the C structs for callers
that hold pointers instead of tensors.

``stream``: a ``torch.cuda.Stream``, a raw ``cudaStream_t`` value, or None for torch's current stream.
``workspace``: a :class:`Workspace`, which a program keeps and hands to one call after the other on one
stream; without one, a call takes fresh memory from torch, and nobody can ask afterwards (:func:`bcast_serve_status`)
whether a wait in it ran out and left its output incomplete.

The operators go forward only: inputs may require gradients, results have none.
"""
from __future__ import annotations

import ctypes

import torch

from . import bcast as _B
from .bcast import BCAST_ERR_CAPACITY, BCAST_ERR_INVAL, BCAST_OK, BcastError, _check, _lib

try:
    from . import _serve_native as _native
except ImportError as _e:
    raise ImportError("the extension module _serve_native does not load: build it with "
                      f"`python -m paper_1603_06809_b200.build` ({_e})") from _e

BCAST_SERVE_BF16, BCAST_SERVE_FP16, BCAST_SERVE_FP32 = 0, 1, 2
BCAST_SERVE_STATUS_BYTES = 256

#: every symbol ``include/bcast_serve.h`` declares
SYMBOLS = ("bcast_serve_linear", "bcast_serve_linear_workspace", "bcast_serve_attn", "bcast_serve_attn_workspace",
           "bcast_serve_verify", "bcast_serve_verify_workspace", "bcast_serve_append", "bcast_serve_logprobs", "bcast_serve_pack4",
           "bcast_serve_unpack4", "bcast_serve_linear4", "bcast_serve_linear4_workspace", "bcast_serve_status")

_vp, _i32, _i64, _u64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_float
_s2, _s3 = _i64 * 2, _i64 * 3


class LinearArgs(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("num_adapters", _i32), ("rank", _i32), ("tokens", _i64), ("k", _i64), ("n", _i64),
                ("x", _vp), ("weight", _vp), ("bias", _vp), ("lora_a", _vp), ("lora_b", _vp), ("adapter", _vp), ("scale", _vp),
                ("y", _vp), ("x_stride", _i64), ("weight_stride", _i64), ("y_stride", _i64), ("lora_a_stride", _s2),
                ("lora_b_stride", _s2), ("workspace", _vp), ("workspace_bytes", _u64)]


class AttnArgs(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("batch", _i32), ("new_tokens", _i32), ("q_heads", _i32), ("kv_heads", _i32), ("dim", _i32),
                ("page_size", _i32), ("scale", _f32), ("prefix_len", _i64), ("own_cap", _i64), ("num_pages", _i64),
                ("q", _vp), ("prefix_k", _vp), ("prefix_v", _vp), ("own_k", _vp), ("own_v", _vp), ("own_len", _vp),
                ("page_table", _vp), ("out", _vp), ("lse", _vp), ("q_stride", _s3), ("out_stride", _s3),
                ("prefix_k_stride", _s2), ("prefix_v_stride", _s2), ("own_k_stride", _s3), ("own_v_stride", _s3),
                ("page_table_stride", _i64), ("workspace", _vp), ("workspace_bytes", _u64)]


class VerifyArgs(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("batch", _i32), ("drafts", _i32), ("vocab", _i64), ("logits", _vp), ("draft_probs", _vp),
                ("uniforms", _vp), ("noise", _vp), ("temperature", _vp), ("draft_tokens", _vp), ("accepted", _vp), ("tokens", _vp),
                ("logits_stride", _s2), ("draft_probs_stride", _s2), ("noise_stride", _i64), ("workspace", _vp),
                ("workspace_bytes", _u64)]


class AppendArgs(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("batch", _i32), ("new_tokens", _i32), ("q_heads", _i32), ("kv_heads", _i32), ("dim", _i32),
                ("page_size", _i32), ("rot", _i32), ("interleaved", _i32), ("axes", _i32), ("eps", _f32), ("own_cap", _i64),
                ("num_pages", _i64), ("first", _i64), ("q", _vp), ("k", _vp), ("v", _vp), ("q_norm", _vp), ("k_norm", _vp),
                ("inv_freq", _vp), ("positions", _vp), ("axis", _vp), ("own_len", _vp), ("new_len", _vp), ("page_table", _vp),
                ("out", _vp), ("own_k", _vp), ("own_v", _vp), ("q_stride", _s3), ("k_stride", _s3), ("v_stride", _s3),
                ("out_stride", _s3), ("own_k_stride", _s3), ("own_v_stride", _s3), ("positions_stride", _s2), ("page_table_stride", _i64)]


class LogprobsArgs(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("top", _i32), ("rows", _i64), ("vocab", _i64), ("logits", _vp), ("tokens", _vp), ("logprobs", _vp),
                ("entropy", _vp), ("top_logprobs", _vp), ("top_tokens", _vp), ("logits_stride", _i64)]


class Pack4Args(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("rows", _i64), ("k", _i64), ("values", _vp), ("codes", _vp), ("scales", _vp), ("values_stride", _i64),
                ("codes_stride", _i64)]


class Linear4Args(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("tokens", _i64), ("k", _i64), ("n", _i64), ("x", _vp), ("bias", _vp), ("codes", _vp), ("scales", _vp),
                ("y", _vp), ("x_stride", _i64), ("codes_stride", _i64), ("y_stride", _i64), ("workspace", _vp), ("workspace_bytes", _u64)]


for _name, _args, _scratch in (("linear", LinearArgs, True), ("attn", AttnArgs, True), ("verify", VerifyArgs, True), ("append", AppendArgs, False),
                               ("logprobs", LogprobsArgs, False), ("pack4", Pack4Args, False), ("unpack4", Pack4Args, False),
                               ("linear4", Linear4Args, True)):
    _f = getattr(_lib, f"bcast_serve_{_name}")
    _f.restype, _f.argtypes = ctypes.c_int, [ctypes.POINTER(_args), _vp]
    if _scratch:
        _f = getattr(_lib, f"bcast_serve_{_name}_workspace")
        _f.restype, _f.argtypes = _i64, [ctypes.POINTER(_args)]
_lib.bcast_serve_status.restype, _lib.bcast_serve_status.argtypes = ctypes.c_int, [_vp, _vp]


class Workspace:
    """Device scratch that grows to what the calls need.  Calls that share one must be ordered on the
    GPU: use one per stream.  What its status word holds stays when it grows.

    Calls may be captured into a CUDA graph with a workspace that is large enough by then (:meth:`reserve`, or
    the same calls once before): it does not grow during a capture (``BCAST_ERR_CAPACITY``).  A larger call
    afterwards leaves the graph the memory it was captured with; keep the workspace as long as the graph."""

    def __init__(self, device="cuda", nbytes: int = 0):
        self.device = torch.device(device)
        self._t, self._of = None, 0
        self._captured, self._kept = False, []            # is a graph using _t; what graphs use of what it was before
        if nbytes:
            self.reserve(nbytes)

    def reserve(self, nbytes: int, stream=None) -> torch.Tensor:
        """Memory of at least ``nbytes``; its status word is zero at first."""
        if self._t is None or self._t.numel() < nbytes:
            with torch.cuda.stream(_torch_stream(stream, self.device)):
                here, old = torch.cuda.current_stream(self.device), self._t
                if torch.cuda.is_current_stream_capturing():
                    raise BcastError(BCAST_ERR_CAPACITY, f"serve.Workspace.reserve ({nbytes} bytes have to be there before the capture)")
                new = torch.empty(max(int(nbytes * 1.25), 1 << 16), dtype=torch.uint8, device=self.device)
                status = new[:BCAST_SERVE_STATUS_BYTES]
                if old is None:
                    status.zero_()
                else:
                    # the old memory goes back to torch's allocator, which reuses it in the order of its streams
                    status.copy_(old[:BCAST_SERVE_STATUS_BYTES])
                    if self._of != here.cuda_stream:
                        old.record_stream(here)
                    if self._captured:
                        self._kept.append(old)
                self._t, self._of, self._captured = new, here.cuda_stream, False
        return self._t


class _Fresh:
    """The memory of one call.  In a capture it is the graph's: torch keeps what such a call allocates for the graph
    alone, and zeroing the status word is part of it."""

    def __init__(self, device):
        self.device, self._t, self._of = device, None, 0

    def reserve(self, nbytes: int, stream=None) -> None:
        with torch.cuda.stream(_torch_stream(stream, self.device)):
            self._t = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            self._t[:BCAST_SERVE_STATUS_BYTES].zero_()
            self._of = torch.cuda.current_stream(self.device).cuda_stream


def _torch_stream(stream, device):
    if stream is None:
        return torch.cuda.current_stream(device)
    if isinstance(stream, torch.cuda.Stream):
        return stream
    return torch.cuda.ExternalStream(int(stream), device=device) if int(stream) else torch.cuda.default_stream(device)


def _strides(t: torch.Tensor, n: int):
    """Strides of the first ``n`` dimensions as the calls pass them on."""
    return _native.strides(t, n)


def _raw(stream) -> int:
    return -1 if stream is None else int(getattr(stream, "cuda_stream", stream))


def _result(where: str, code: int, result):
    if code == BCAST_OK:
        return result
    raise BcastError(code, f"{where} ({result})" if code == BCAST_ERR_INVAL and result else where)


def _call(where: str, native, device, workspace, stream, *tensors):
    """The native call, once more with a larger workspace where it asks for one."""
    raw = _raw(stream)
    if workspace is None:
        workspace = _Fresh(device)
    code, result, captured = native(*tensors, workspace._t, workspace._of, raw)
    if code == BCAST_ERR_CAPACITY:
        workspace.reserve(result, stream)
        code, result, captured = native(*tensors, workspace._t, workspace._of, raw)
    if captured:
        workspace._captured = True
    return _result(where, code, result)


def bcast_serve_linear(x, weight, *, bias=None, lora_a=None, lora_b=None, adapter=None, scale=None, out=None, workspace=None,
                       stream=None):
    """``x`` [T, k], ``weight`` [n, k], ``bias`` [n], ``lora_a`` [L, R, k], ``lora_b`` [L, n, R], ``adapter`` [T] int32
    (-1: none), ``scale`` [L] float32.  Returns y [T, n]: ``x @ weight.T + bias`` plus, token by token,
    ``scale[a] * lora_b[a] @ (lora_a[a] @ x[t])``."""
    return _call("bcast_serve_linear", _native.linear, x.device, workspace, stream, x, weight, bias, lora_a, lora_b, adapter, scale, out)


def bcast_serve_attn(q, prefix_k, prefix_v, own_k, own_v, own_len, *, page_table=None, scale=None, out=None, lse=None,
                     workspace=None, stream=None):
    """``q`` [B, n, HQ, D]; ``prefix_k``/``prefix_v`` [P, H, D], shared by all requests; the requests' own tokens in rows
    (``own_k``/``own_v`` [B, S, H, D]) or in pages ([pages, page_size, H, D] with ``page_table`` [B, pages per request]
    int32); ``own_len`` [B] int32, the own tokens in the cache, the n new ones among them.  ``scale`` defaults to
    D ** -0.5.  Returns out [B, n, HQ, D]; ``lse`` [B, n, HQ] float32 is filled if given."""
    return _call("bcast_serve_attn", _native.attn, q.device, workspace, stream, q, prefix_k, prefix_v, own_k, own_v, own_len, page_table,
                 scale, out, lse)


def bcast_serve_verify(logits, draft_probs, draft_tokens, uniforms, noise, temperature, *, accepted=None, tokens=None,
                       workspace=None, stream=None):
    """``logits`` [B, n + 1, V] of the target; ``draft_probs`` [B, n, V] float32 and ``draft_tokens`` [B, n] int32 of the
    draft; ``uniforms`` [B, n], ``noise`` [B, V] (unit exponential) and ``temperature`` [B], all float32.  Returns
    (accepted [B], tokens [B, n + 1]), both int32: the accepted drafts, the token after them, then -1."""
    return _call("bcast_serve_verify", _native.verify, logits.device, workspace, stream, logits, draft_probs, draft_tokens, uniforms, noise,
                 temperature, accepted, tokens)


def bcast_serve_append(q, k, v, own_k, own_v, own_len, *, page_table=None, new_len=None, first=0, positions=None, inv_freq=None, axis=None,
                       interleaved=False, q_norm=None, k_norm=None, eps=1e-6, out=None, stream=None):
    """``q`` [B, n, HQ, D] (or None), ``k``/``v`` [B, n, H, D] of the n newest tokens of every request; the caches, ``own_len``
    and ``page_table`` as :func:`bcast_serve_attn` takes them afterwards, the new tokens counted in ``own_len`` already.
    Queries and keys are normed with ``q_norm``/``k_norm`` [D] and rotated by ``inv_freq`` [rot / 2] float32, where
    given, at ``first`` + place in the cache or at ``positions`` [B, n] or [B, n, axes] int32 (``axis`` [rot / 2] int32: the axis
    of each pair); keys and values go into the caches.  ``new_len`` [B] int32: how many of the n are there, at the end.
    Returns the queries (``out``, which may be ``q``), None without ``q``."""
    code, result, _ = _native.append(q, k, v, own_k, own_v, own_len, page_table, new_len, first, positions, inv_freq, axis, interleaved, q_norm,
                                     k_norm, eps, out, _raw(stream))
    return _result("bcast_serve_append", code, result)


def bcast_serve_logprobs(logits, tokens, *, top=0, logprobs=None, entropy=None, top_tokens=None, top_logprobs=None, stream=None):
    """``logits`` [T, V], ``tokens`` [T] int32.  Returns (logprobs [T], entropy [T], top_tokens [T, top] int32, top_logprobs
    [T, top]), float32 where nothing else is said: the given tokens' log probabilities, and the ``top`` most probable tokens."""
    code, result, _ = _native.logprobs(logits, tokens, top, logprobs, entropy, top_tokens, top_logprobs, _raw(stream))
    return _result("bcast_serve_logprobs", code, result)


def bcast_serve_pack4(x, *, codes=None, scales=None, stream=None):
    """``x`` [rows, k] bf16, fp16 or fp32, k a multiple of 32.  Returns (codes [rows, k / 2], scales [ceil(rows / 128),
    ceil(k / 128), 32, 4, 4]), both uint8: microscaled 4-bit numbers."""
    code, result, _ = _native.pack4(x, codes, scales, _raw(stream))
    return _result("bcast_serve_pack4", code, result)


def bcast_serve_unpack4(codes, scales, dtype=torch.bfloat16, *, out=None, stream=None):
    """The numbers [rows, k] that ``codes`` and ``scales`` stand for, in ``dtype``."""
    code, result, _ = _native.unpack4(codes, scales, dtype, out, _raw(stream))
    return _result("bcast_serve_unpack4", code, result)


def bcast_serve_linear4(x, codes, scales, *, bias=None, out=None, workspace=None, stream=None):
    """``x`` [T, k]; ``codes``, ``scales`` of a weight [n, k] as :func:`bcast_serve_pack4` makes them; ``bias`` [n].  Returns
    y [T, n]: x, packed in the same way, times the weight."""
    return _call("bcast_serve_linear4", _native.linear4, x.device, workspace, stream, x, codes, scales, bias, out)


def bcast_serve_status(workspace: Workspace, stream=None) -> None:
    """Waits for ``stream`` and raises ``BcastError`` (``BCAST_ERR_TIMEOUT``) if a kernel that used this
    workspace gave up on one of its bounded waits; returns None otherwise."""
    mem = workspace._t
    if mem is None:                                       # no call used it yet
        return _torch_stream(stream, workspace.device).synchronize()
    raw = torch.cuda.current_stream(workspace.device).cuda_stream if stream is None else _B._stream_ptr(stream)
    with torch.cuda.device(mem.device):
        for code in [_lib.bcast_serve_status(m.data_ptr(), raw) for m in (mem, *workspace._kept)]:
            _check(code, "bcast_serve_status")
