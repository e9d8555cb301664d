"""ctypes binding of ``include/bcast_serve.h``: same names, torch tensors in place of pointers.

The functions check that the tensors have the shapes and types of one call, describe them to the C
entry point of the same name (which checks ranges, alignment and strides) and return what it writes;
nothing is computed in Python.  Tensors are taken with their strides and are never copied; the
innermost dimension has to be contiguous.

``stream``: a ``torch.cuda.Stream``, a raw ``cudaStream_t`` value, or None for torch's current stream.
``workspace``: a :class:`Workspace`, which a program keeps and hands to one call after the other on one
stream; without one, a call takes fresh memory from torch.
"""
from __future__ import annotations

import ctypes

import torch

from . import bcast as _B
from .bcast import BCAST_ERR_INVAL, BcastError, _check, _lib

BCAST_SERVE_BF16, BCAST_SERVE_FP16, BCAST_SERVE_FP32 = 0, 1, 2
BCAST_SERVE_STATUS_BYTES = 256

_DTYPE = {torch.bfloat16: BCAST_SERVE_BF16, torch.float16: BCAST_SERVE_FP16, torch.float32: BCAST_SERVE_FP32}

#: every symbol ``include/bcast_serve.h`` declares
SYMBOLS = ("bcast_serve_linear", "bcast_serve_linear_workspace", "bcast_serve_attn", "bcast_serve_attn_workspace",
           "bcast_serve_verify", "bcast_serve_verify_workspace", "bcast_serve_status")

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


for _name, _args in (("linear", LinearArgs), ("attn", AttnArgs), ("verify", VerifyArgs)):
    _f = getattr(_lib, f"bcast_serve_{_name}")
    _f.restype, _f.argtypes = ctypes.c_int, [ctypes.POINTER(_args), _vp]
    _f = getattr(_lib, f"bcast_serve_{_name}_workspace")
    _f.restype, _f.argtypes = _i64, [ctypes.POINTER(_args)]
_lib.bcast_serve_status.restype, _lib.bcast_serve_status.argtypes = ctypes.c_int, [_vp, _vp]


class Workspace:
    """Device scratch that grows to what the calls need.  Calls that share one must be ordered on the
    GPU: use one per stream."""

    def __init__(self, device="cuda", nbytes: int = 0):
        self.device = torch.device(device)
        self._t, self._of = None, None
        if nbytes:
            self.reserve(nbytes)

    def reserve(self, nbytes: int, stream=None) -> torch.Tensor:
        """Memory of at least ``nbytes`` whose status word has been zeroed."""
        if self._t is None or self._t.numel() < nbytes:
            with torch.cuda.stream(_torch_stream(stream, self.device)):
                # the old memory goes back to torch's allocator, which reuses it in the order of its streams
                self._t = torch.empty(max(int(nbytes * 1.25), 1 << 16), dtype=torch.uint8, device=self.device)
                self._t[:BCAST_SERVE_STATUS_BYTES].zero_()
                self._of = torch.cuda.current_stream(self.device).cuda_stream
        return self._t

    def used_on(self, raw: int) -> None:
        """The memory is in use on stream ``raw``, which need not be the one it was allocated on."""
        if raw != self._of:
            self._t.record_stream(_torch_stream(raw, self._t.device))


def _torch_stream(stream, device):
    if stream is None:
        return torch.cuda.current_stream(device)
    if isinstance(stream, torch.cuda.Stream):
        return stream
    return torch.cuda.ExternalStream(int(stream), device=device) if int(stream) else torch.cuda.default_stream(device)


def _need(ok: bool, where: str, what: str) -> None:
    if not ok:
        raise BcastError(BCAST_ERR_INVAL, f"{where} ({what})")


def _strides(t: torch.Tensor, n: int):
    """Strides of the first ``n`` dimensions; where a dimension has one entry its stride means nothing and
    is given as that of a contiguous array."""
    st, sh = t.stride(), t.shape
    if 1 not in sh[:n]:
        return st[:n]
    out, run = [], 1
    for i in range(len(sh) - 1, -1, -1):
        s = run if sh[i] == 1 else st[i]
        run = max(run, -(-s * sh[i] // 8) * 8)
        out.append(s)
    return tuple(out[::-1][:n])


def _array(t, where: str, name: str, dtype, shape, device) -> None:
    """One tensor against what the call expects of it."""
    if t.dtype is not dtype or t.shape != shape or t.device != device or (shape and shape[-1] > 1 and t.stride(-1) != 1):
        raise BcastError(BCAST_ERR_INVAL, f"{where} ({name}: {tuple(t.shape)} {t.dtype} on {t.device} with strides {t.stride()}, "
                                          f"expected {tuple(shape)} {dtype} on {device}, last dimension contiguous)")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _call(name: str, args, device, workspace, stream) -> None:
    need = getattr(_lib, name + "_workspace")(args)
    if need < 0:
        raise BcastError(int(need), name)
    raw = torch.cuda.current_stream(device).cuda_stream if stream is None else int(getattr(stream, "cuda_stream", stream))
    if workspace is None:
        workspace = Workspace(device)
    mem = workspace.reserve(need, stream)
    args.workspace, args.workspace_bytes = mem.data_ptr(), mem.numel()
    if torch.cuda.current_device() == device.index:
        code = getattr(_lib, name)(args, raw)
    else:
        with torch.cuda.device(device):
            code = getattr(_lib, name)(args, raw)
    workspace.used_on(raw)
    _check(code, name)


def _out(out, where, name, shape, dtype, device, stream):
    if out is None:
        with torch.cuda.stream(_torch_stream(stream, device)) if stream is not None else _nothing:
            return torch.empty(shape, dtype=dtype, device=device)
    _array(out, where, name, dtype, torch.Size(shape), device)
    return out


class _Nothing:
    def __enter__(self):
        return None

    def __exit__(self, *_):
        return False


_nothing = _Nothing()


def bcast_serve_linear(x, weight, *, bias=None, lora_a=None, lora_b=None, adapter=None, scale=None, out=None, workspace=None,
                       stream=None):
    """``x`` [T, k], ``weight`` [n, k], ``bias`` [n], ``lora_a`` [L, R, k], ``lora_b`` [L, n, R], ``adapter`` [T] int32
    (-1: none), ``scale`` [L] float32.  Returns y [T, n]: ``x @ weight.T + bias`` plus, token by token,
    ``scale[a] * lora_b[a] @ (lora_a[a] @ x[t])``."""
    where = "bcast_serve_linear"
    dt, dev = x.dtype, x.device
    _need(x.dim() == 2 and weight.dim() == 2, where, "x and weight have two dimensions")
    _need(dt in (torch.bfloat16, torch.float16), where, f"type {dt}")
    _need(dev.type == "cuda", where, "tensors on a CUDA device")
    T, K = x.shape
    N = weight.shape[0]
    _array(x, where, "x", dt, x.shape, dev)
    _array(weight, where, "weight", dt, torch.Size((N, K)), dev)
    if bias is not None:
        _array(bias, where, "bias", dt, torch.Size((N,)), dev)
    L = R = 0
    as_ = bs = (0, 0)
    if lora_a is not None:
        _need(lora_b is not None and adapter is not None and scale is not None, where, "lora_a, lora_b, adapter and scale go together")
        _need(lora_a.dim() == 3, where, "lora_a has three dimensions")
        L, R = lora_a.shape[:2]
        _array(lora_a, where, "lora_a", dt, torch.Size((L, R, K)), dev)
        _array(lora_b, where, "lora_b", dt, torch.Size((L, N, R)), dev)
        _array(adapter, where, "adapter", torch.int32, torch.Size((T,)), dev)
        _array(scale, where, "scale", torch.float32, torch.Size((L,)), dev)
        as_, bs = _strides(lora_a, 2), _strides(lora_b, 2)
    else:
        _need(lora_b is None and adapter is None and scale is None, where, "lora_a, lora_b, adapter and scale go together")
    y = _out(out, where, "out", (T, N), dt, dev, stream)
    args = LinearArgs(_DTYPE[dt], L, R, T, K, N, x.data_ptr(), weight.data_ptr(), _ptr(bias), _ptr(lora_a), _ptr(lora_b),
                      _ptr(adapter), _ptr(scale), y.data_ptr(), _strides(x, 1)[0], _strides(weight, 1)[0], _strides(y, 1)[0],
                      _s2(*as_), _s2(*bs), None, 0)
    _call(where, args, dev, workspace, stream)
    return y


def bcast_serve_attn(q, prefix_k, prefix_v, own_k, own_v, own_len, *, page_table=None, scale=None, out=None, lse=None,
                     workspace=None, stream=None):
    """``q`` [B, n, HQ, D]; ``prefix_k``/``prefix_v`` [P, H, D], shared by all requests; the requests' own tokens in rows
    (``own_k``/``own_v`` [B, S, H, D]) or in pages ([pages, page_size, H, D] with ``page_table`` [B, pages per request]
    int32); ``own_len`` [B] int32, the own tokens in the cache, the n new ones among them.  ``scale`` defaults to
    D ** -0.5.  Returns out [B, n, HQ, D]; ``lse`` [B, n, HQ] float32 is filled if given."""
    where = "bcast_serve_attn"
    dt, dev = q.dtype, q.device
    _need(q.dim() == 4 and prefix_k.dim() == 3 and own_k.dim() == 4, where, "q and own_k have four dimensions, prefix_k three")
    _need(dt in (torch.bfloat16, torch.float16), where, f"type {dt}")
    _need(dev.type == "cuda", where, "tensors on a CUDA device")
    B, n, HQ, D = q.shape
    P, H = prefix_k.shape[:2]
    _array(q, where, "q", dt, q.shape, dev)
    kv = torch.Size((P, H, D))
    _array(prefix_k, where, "prefix_k", dt, kv, dev)
    _array(prefix_v, where, "prefix_v", dt, kv, dev)
    own = torch.Size((own_k.shape[0] if page_table is not None else B, own_k.shape[1], H, D))
    _array(own_k, where, "own_k", dt, own, dev)
    _array(own_v, where, "own_v", dt, own, dev)
    _array(own_len, where, "own_len", torch.int32, torch.Size((B,)), dev)
    page = pages = pts = 0
    cap = own[1]
    if page_table is not None:
        _need(page_table.dim() == 2 and own[1] >= 1, where, "page_table has two dimensions, a page at least one token")
        page, pages = own[1], own[0]
        cap = page_table.shape[1] * page
        _array(page_table, where, "page_table", torch.int32, torch.Size((B, page_table.shape[1])), dev)
        pts = _strides(page_table, 1)[0]
    if lse is not None:
        _array(lse, where, "lse", torch.float32, torch.Size((B, n, HQ)), dev)
        _need(lse.is_contiguous(), where, "lse is contiguous")
    o = _out(out, where, "out", (B, n, HQ, D), dt, dev, stream)
    args = AttnArgs(_DTYPE[dt], B, n, HQ, H, D, page, D ** -0.5 if scale is None else scale, P, cap, pages, q.data_ptr(),
                    prefix_k.data_ptr(), prefix_v.data_ptr(), own_k.data_ptr(), own_v.data_ptr(), own_len.data_ptr(),
                    _ptr(page_table), o.data_ptr(), _ptr(lse), _s3(*_strides(q, 3)), _s3(*_strides(o, 3)),
                    _s2(*_strides(prefix_k, 2)), _s2(*_strides(prefix_v, 2)), _s3(*_strides(own_k, 3)), _s3(*_strides(own_v, 3)),
                    pts, None, 0)
    _call(where, args, dev, workspace, stream)
    return o


def bcast_serve_verify(logits, draft_probs, draft_tokens, uniforms, noise, temperature, *, accepted=None, tokens=None,
                       workspace=None, stream=None):
    """``logits`` [B, n + 1, V] of the target; ``draft_probs`` [B, n, V] float32 and ``draft_tokens`` [B, n] int32 of the
    draft; ``uniforms`` [B, n], ``noise`` [B, V] (unit exponential) and ``temperature`` [B], all float32.  Returns
    (accepted [B], tokens [B, n + 1]), both int32: the accepted drafts, the token after them, then -1."""
    where = "bcast_serve_verify"
    dt, dev = logits.dtype, logits.device
    _need(logits.dim() == 3 and logits.shape[1] >= 1, where, "logits has three dimensions and at least one row")
    _need(dt in _DTYPE, where, f"type {dt}")
    _need(dev.type == "cuda", where, "tensors on a CUDA device")
    B, n1, V = logits.shape
    n = n1 - 1
    f32 = torch.float32
    _array(logits, where, "logits", dt, logits.shape, dev)
    _array(draft_probs, where, "draft_probs", f32, torch.Size((B, n, V)), dev)
    bn = torch.Size((B, n))
    _array(draft_tokens, where, "draft_tokens", torch.int32, bn, dev)
    _array(uniforms, where, "uniforms", f32, bn, dev)
    _need(draft_tokens.is_contiguous() and uniforms.is_contiguous(), where, "draft_tokens and uniforms are contiguous")
    _array(noise, where, "noise", f32, torch.Size((B, V)), dev)
    _array(temperature, where, "temperature", f32, torch.Size((B,)), dev)
    accepted = _out(accepted, where, "accepted", (B,), torch.int32, dev, stream)
    tokens = _out(tokens, where, "tokens", (B, n1), torch.int32, dev, stream)
    _need(tokens.is_contiguous(), where, "tokens is contiguous")
    args = VerifyArgs(_DTYPE[dt], B, n, V, logits.data_ptr(), draft_probs.data_ptr(), uniforms.data_ptr(), noise.data_ptr(),
                      temperature.data_ptr(), draft_tokens.data_ptr(), accepted.data_ptr(), tokens.data_ptr(),
                      _s2(*_strides(logits, 2)), _s2(*_strides(draft_probs, 2)), _strides(noise, 1)[0], None, 0)
    _call(where, args, dev, workspace, stream)
    return accepted, tokens


def bcast_serve_status(workspace: Workspace, stream=None) -> None:
    """Waits for ``stream`` and raises ``BcastError`` (``BCAST_ERR_TIMEOUT``) if a kernel that used this
    workspace gave up on one of its bounded waits; returns None otherwise."""
    mem = workspace.reserve(BCAST_SERVE_STATUS_BYTES)
    raw = torch.cuda.current_stream(workspace.device).cuda_stream if stream is None else _B._stream_ptr(stream)
    with torch.cuda.device(mem.device):
        _check(_lib.bcast_serve_status(mem.data_ptr(), raw), "bcast_serve_status")
