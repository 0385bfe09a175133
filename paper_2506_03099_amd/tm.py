"""ctypes binding of ``libtm.so`` (the C ABI in ``include/tm.h``).

Argument marshalling only: torch tensors supply device pointers, the current
HIP stream supplies the stream (or the caller, who orders it behind what makes the inputs and ahead of
what uses the outputs), and every step of the computation runs in the
library's HIP kernels. The binding raises if the library has not been built;
there is no other implementation to fall back to.

Function names match the C entry points.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libtm.so")

TM_OK = 0
TM_E_ARG = -1
TM_E_SHAPE = -2
TM_E_DTYPE = -3
TM_E_ORDER = -4
TM_E_CAPACITY = -5
TM_E_DEVICE = -6
TM_F32 = 0
TM_BF16 = 1
TM_MAX_WINDOW = 12
TM_MAX_AUDIO_STREAMS = 32

STATUS_NAMES = {0: "TM_OK", -1: "TM_E_ARG", -2: "TM_E_SHAPE", -3: "TM_E_DTYPE",
                -4: "TM_E_ORDER", -5: "TM_E_CAPACITY", -6: "TM_E_DEVICE"}

_TORCH_DTYPE = {TM_F32: torch.float32, TM_BF16: torch.bfloat16}
_BF16 = torch.bfloat16
_DTYPE_CODE = {torch.float32: TM_F32, torch.bfloat16: TM_BF16, "f32": TM_F32, "bf16": TM_BF16}


class tm_attn_desc(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("tokens_per_frame", ctypes.c_int32),
        ("chunk_frames", ctypes.c_int32),
        ("ref_frames", ctypes.c_int32),
        ("window", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("softmax_scale", ctypes.c_float),
    ]

    @property
    def torch_dtype(self):
        return _TORCH_DTYPE[self.dtype]


class tm_audio_desc(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("tokens_per_frame", ctypes.c_int32),
        ("audio_per_frame", ctypes.c_int32),
        ("audio_frames", ctypes.c_int32),
        ("streams", ctypes.c_int32),
        ("half_window", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("softmax_scale", ctypes.c_float),
    ]


class tm_rope_desc(ctypes.Structure):
    _fields_ = [
        ("head_dim", ctypes.c_int32),
        ("frames", ctypes.c_int32),
        ("grid_h", ctypes.c_int32),
        ("grid_w", ctypes.c_int32),
        ("pairs_t", ctypes.c_int32),
        ("pairs_h", ctypes.c_int32),
        ("pairs_w", ctypes.c_int32),
        ("split_half", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("theta", ctypes.c_float),
    ]


TM_NORM_NONE, TM_NORM_LAYER, TM_NORM_RMS = 0, 1, 2
TM_ACT_NONE, TM_ACT_GELU, TM_ACT_SILU = 0, 1, 2
_NORM_CODE = {"none": TM_NORM_NONE, None: TM_NORM_NONE, "layer": TM_NORM_LAYER, "rms": TM_NORM_RMS}
_ACT_CODE = {"none": TM_ACT_NONE, None: TM_ACT_NONE, "gelu": TM_ACT_GELU, "silu": TM_ACT_SILU}


class tm_block_norm_desc(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("width", ctypes.c_int32),
        ("pre", ctypes.c_int32),
        ("post", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("stream_dtype", ctypes.c_int32),
        ("groups", ctypes.c_int32),
        ("group_tokens", ctypes.c_int32),
        ("eps", ctypes.c_float),
    ]


class tm_linear_desc(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("in_width", ctypes.c_int32),
        ("out_width", ctypes.c_int32),
        ("act", ctypes.c_int32),
        ("out_dtype", ctypes.c_int32),
        ("groups", ctypes.c_int32),
        ("group_tokens", ctypes.c_int32),
    ]


class TMError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    """Load ``libtm.so`` (built by ``paper_2506_03099_amd.build``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with "
                               "`python -m paper_2506_03099_amd.build`")
        L = ctypes.CDLL(_LIB_PATH)
        P = ctypes.c_void_p
        D = ctypes.POINTER(tm_attn_desc)
        AD = ctypes.POINTER(tm_audio_desc)
        RD = ctypes.POINTER(tm_rope_desc)
        ND = ctypes.POINTER(tm_block_norm_desc)
        LD = ctypes.POINTER(tm_linear_desc)
        rope = [RD, P, ctypes.c_int32, ctypes.c_int32, ctypes.c_int64, P, ctypes.c_int32, P,
                ctypes.c_int32, P, P, P]
        sig = {
            "tm_kv_cache_tokens": (ctypes.c_int64, [D]),
            "tm_kv_cache_bytes": (ctypes.c_size_t, [D]),
            "tm_kv_cache_create": (ctypes.c_int, [D, P, P, ctypes.POINTER(P)]),
            "tm_kv_cache_destroy": (None, [P]),
            "tm_kv_cache_reset": (ctypes.c_int, [P]),
            "tm_kv_cache_locate": (ctypes.c_int, [P, ctypes.c_int32,
                                                  ctypes.POINTER(ctypes.c_int32),
                                                  ctypes.POINTER(ctypes.c_int32)]),
            "tm_kv_cache_latest": (ctypes.c_int32, [P]),
            "tm_kv_append": (ctypes.c_int, [P, ctypes.c_int32, P, P, ctypes.c_int32, P]),
            "tm_qkv_produce": (ctypes.c_int, [P, ctypes.c_int32, P, P, P, P, P, ctypes.c_float,
                                              P, ctypes.c_int32, P]),
            "tm_sparse_causal_attn_fwd": (ctypes.c_int, [D, P, ctypes.c_int32, P, P, P,
                                                         ctypes.c_int32, P, P, P]),
            "tm_sparse_causal_attn_fwd_f32out": (ctypes.c_int, [D, P, ctypes.c_int32, P, P, P,
                                                                ctypes.c_int32, P, P, P]),
            "tm_sparse_causal_attn_fwd_workspace": (ctypes.c_size_t, [D, ctypes.c_int32, P,
                                                                      ctypes.c_int32]),
            "tm_sparse_causal_attn_fwd_ws": (ctypes.c_int, [D, P, ctypes.c_int32, P, P, P,
                                                            ctypes.c_int32, P, ctypes.c_int32, P, P,
                                                            ctypes.c_size_t, P]),
            "tm_allowed_pairs": (ctypes.c_int64, [D, ctypes.c_int32, P, ctypes.c_int32]),
            "tm_audio_cross_attn_fwd": (ctypes.c_int, [AD, P, ctypes.c_int32, ctypes.c_int32, P, P,
                                                       P, P, P]),
            "tm_audio_cross_attn_fwd_f32out": (ctypes.c_int, [AD, P, ctypes.c_int32,
                                                              ctypes.c_int32, P, P, P, P, P]),
            "tm_sparse_causal_attn_bwd": (ctypes.c_int, [D, ctypes.c_int32, P, P, P, P, P, P, P,
                                                         P, P, P, P]),
            "tm_sparse_causal_attn_bwd_workspace": (ctypes.c_size_t, [D, ctypes.c_int32]),
            "tm_sparse_causal_attn_bwd_ws": (ctypes.c_int, [D, ctypes.c_int32, P, P, P, P, P, P, P,
                                                            P, P, P, P, ctypes.c_size_t, P]),
            "tm_sparse_causal_attn_bwd_noalloc": (ctypes.c_int, [D, ctypes.c_int32, P, P, P, P, P,
                                                                 P, P, P, P, P]),
            "tm_rope3d_table_bytes": (ctypes.c_size_t, [RD]),
            "tm_rope3d_table": (ctypes.c_int, [RD, P, P]),
            "tm_rope3d_fwd": (ctypes.c_int, rope),
            "tm_rope3d_bwd": (ctypes.c_int, rope),
            "tm_kv8_cache_tokens": (ctypes.c_int64, [D]),
            "tm_kv8_cache_bytes": (ctypes.c_size_t, [D, ctypes.c_int32]),
            "tm_kv8_cache_create": (ctypes.c_int, [D, ctypes.c_int32, P, ctypes.POINTER(P)]),
            "tm_kv8_cache_destroy": (None, [P]),
            "tm_kv8_cache_reset": (ctypes.c_int, [P]),
            "tm_kv8_cache_latest": (ctypes.c_int32, [P]),
            "tm_kv8_cache_locate": (ctypes.c_int, [P, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32),
                                                   ctypes.POINTER(ctypes.c_int32)]),
            "tm_kv8_append": (ctypes.c_int, [P, ctypes.c_int32, P, P, ctypes.c_int32, P]),
            "tm_qkv8_produce": (ctypes.c_int, [P, ctypes.c_int32, P, P, P, P, P, ctypes.c_float, RD, P,
                                               ctypes.c_int64, P, ctypes.c_int32, P]),
            "tm_kv8_read": (ctypes.c_int, [P, ctypes.c_int32, P, P, ctypes.c_int32, P]),
            "tm_kv8_attn_workspace": (ctypes.c_size_t, [P, ctypes.c_int32, ctypes.c_int32]),
            "tm_kv8_attn_fwd": (ctypes.c_int, [P, P, ctypes.c_int32, ctypes.c_int32, P, ctypes.c_int32,
                                               P, P, ctypes.c_size_t, P]),
            "tm_block_norm_fwd": (ctypes.c_int, [ND, ctypes.c_int32, ctypes.c_int64] + [P] * 11),
            "tm_block_norm_bwd_workspace": (ctypes.c_size_t, [ND, ctypes.c_int32, ctypes.c_int64]),
            "tm_block_norm_bwd": (ctypes.c_int, [ND, ctypes.c_int32, ctypes.c_int64] + [P] * 18
                                  + [ctypes.c_size_t, P]),
            "tm_linear_fwd_workspace": (ctypes.c_size_t, [LD, ctypes.c_int32]),
            "tm_linear_fwd": (ctypes.c_int, [LD, ctypes.c_int32, ctypes.c_int64] + [P] * 8
                              + [ctypes.c_size_t, P]),
            "tm_linear_bwd_workspace": (ctypes.c_size_t, [LD, ctypes.c_int32, ctypes.c_int64]),
            "tm_linear_bwd": (ctypes.c_int, [LD, ctypes.c_int32, ctypes.c_int64] + [P] * 10
                              + [ctypes.c_size_t, P]),
            "tm_last_error": (ctypes.c_char_p, []),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def tm_last_error() -> str:
    return lib().tm_last_error().decode()


def _check(status: int):
    if status != TM_OK:
        raise TMError(status, tm_last_error())


def _dtype(dtype):
    return _DTYPE_CODE[dtype] if isinstance(dtype, (torch.dtype, str)) else dtype


def make_desc(batch, heads, head_dim, tokens_per_frame, chunk_frames, ref_frames, window,
              dtype, softmax_scale=0.0) -> tm_attn_desc:
    dtype = _dtype(dtype)
    return tm_attn_desc(batch, heads, head_dim, tokens_per_frame, chunk_frames, ref_frames,
                        window, dtype, softmax_scale)


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_cuda:
        raise TMError(TM_E_ARG, "tensor is not on a GPU")
    if not t.is_contiguous():
        raise TMError(TM_E_ARG, "tensor is not contiguous")
    return t.data_ptr()


def _current_stream() -> int:
    # torch.cuda.current_stream() builds a Stream object, 2.6 us of a call that
    # takes 8; the handle alone takes 0.2
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _stream(stream):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


def _new(shape, dtype, device, stream):
    """A tensor that a call on ``stream`` writes. For another stream than the current one it comes from that stream's
    memory, since the current stream may still use what it has freed, and is kept from that stream's later calls until
    the current one is done with it."""
    if stream is None or _stream(stream) == _current_stream():
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(torch.cuda.ExternalStream(_stream(stream), device)):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(torch.cuda.current_stream())
    return t


def _like(t, stream):
    """The same, like ``t``."""
    return torch.empty_like(t) if stream is None else _new(t.shape, t.dtype, t.device, stream)


def tm_kv_cache_tokens(desc: tm_attn_desc) -> int:
    return lib().tm_kv_cache_tokens(ctypes.byref(desc))


def tm_kv_cache_bytes(desc: tm_attn_desc) -> int:
    return lib().tm_kv_cache_bytes(ctypes.byref(desc))


def tm_allowed_pairs(desc: tm_attn_desc, q_chunk: int, cache=None, n_frames: int = 0) -> int:
    h = cache.handle if cache is not None else None
    return lib().tm_allowed_pairs(ctypes.byref(desc), q_chunk, h, n_frames)


class KVCache:
    """A ``tm_kv_cache`` handle together with the torch tensors that own its
    pools: K ``[B, H, capacity, D]``, V ``[B, H, capacity // 64, D, 64]``
    (64-token blocks stored dimension-major)."""

    def __init__(self, desc: tm_attn_desc, device="cuda", k_pool=None, v_pool=None):
        self.desc = desc
        cap = tm_kv_cache_tokens(desc)
        if cap <= 0:
            raise TMError(TM_E_SHAPE, "invalid descriptor")
        B, H, D, dt = desc.batch, desc.heads, desc.head_dim, desc.torch_dtype
        self.k_pool = k_pool if k_pool is not None else torch.empty(
            (B, H, cap, D), dtype=dt, device=device)
        self.v_pool = v_pool if v_pool is not None else torch.empty(
            (B, H, cap // 64, D, 64), dtype=dt, device=device)
        h = ctypes.c_void_p()
        _check(lib().tm_kv_cache_create(ctypes.byref(desc), _ptr(self.k_pool), _ptr(self.v_pool),
                                        ctypes.byref(h)))
        self.handle = h

    @property
    def capacity(self) -> int:
        return self.k_pool.shape[2]

    def close(self):
        if getattr(self, "handle", None) is not None and _lib is not None:
            _lib.tm_kv_cache_destroy(self.handle)
            self.handle = None

    __del__ = close

    def latest(self) -> int:
        return lib().tm_kv_cache_latest(self.handle)

    def locate(self, chunk: int):
        off, n = ctypes.c_int32(), ctypes.c_int32()
        _check(lib().tm_kv_cache_locate(self.handle, chunk, ctypes.byref(off), ctypes.byref(n)))
        return off.value, n.value

    def reset(self):
        _check(lib().tm_kv_cache_reset(self.handle))


def tm_kv_cache_create(desc: tm_attn_desc, device="cuda", k_pool=None, v_pool=None) -> KVCache:
    return KVCache(desc, device, k_pool, v_pool)


def tm_kv_append(cache: KVCache, chunk: int, k, v, n_tok: int | None = None, stream=None):
    """Append chunk ``chunk``'s K/V (``[B, n_tok, H, D]``) to the cache."""
    if n_tok is None:
        n_tok = k.shape[1]
    _check(lib().tm_kv_append(cache.handle, chunk, _ptr(k), _ptr(v), n_tok, _stream(stream)))


def tm_qkv_produce(cache: KVCache, chunk: int, q, k, v, q_gain=None, k_gain=None,
                   eps: float = 0.0, q_out=None, n_tok: int | None = None, stream=None):
    """RMS-normalise the chunk's q and k rows and append k (normalised) and v
    to the cache; returns ``q_out`` (allocated like q if not given)."""
    if n_tok is None:
        n_tok = k.shape[1]
    if q_out is None:
        q_out = _like(q, stream)
    _check(lib().tm_qkv_produce(cache.handle, chunk, _ptr(q), _ptr(k), _ptr(v), _ptr(q_gain),
                                _ptr(k_gain), eps, _ptr(q_out), n_tok, _stream(stream)))
    return q_out


def _workspace(nbytes: int, q, stream: int):
    """A workspace for one call on `stream`: memory of torch's allocator, which
    hands it out again in the order of the current stream once the call has
    returned. None (the call then runs without: the forward over 16-bit keys to the
    same bits, the one over the 8-bit cache and the backward with their fp32 sums in
    another order) where that order does not cover
    the call: q a plain address or on another device than the current one,
    another stream than the current one, or a stream under capture; and where the
    memory is not to be had."""
    if (nbytes == 0 or not isinstance(q, torch.Tensor)
            or q.get_device() != torch._C._cuda_getDevice()
            or stream != _current_stream() or torch.cuda.is_current_stream_capturing()):
        return None
    try:
        return torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    except torch.cuda.OutOfMemoryError:
        return None


def _fwd(desc, q, q_chunk, cache, k, v, n_frames, o, o_f32, lse, stream):
    h = cache.handle if cache is not None else None
    d = ctypes.byref(desc)
    L = lib()
    # (the tensors first: on a host without a GPU there is no stream to ask for)
    pq, pk, pv, po, pl = _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse)
    stream = _stream(stream)
    ws, n = None, 0
    if desc.dtype == TM_BF16:
        n = L.tm_sparse_causal_attn_fwd_workspace(d, q_chunk, h, n_frames)
        if n:
            ws = _workspace(n, q, stream)
    _check(L.tm_sparse_causal_attn_fwd_ws(d, pq, q_chunk, h, pk, pv, n_frames, po, o_f32, pl, _ptr(ws), n,
                                          stream))
    return o


def tm_sparse_causal_attn_fwd(desc: tm_attn_desc, q, q_chunk: int, cache: KVCache | None = None,
                              k=None, v=None, n_frames: int = 0, o=None, lse=None,
                              stream=None):
    """Sparse causal attention; returns ``o`` (allocated like q if not given)."""
    if o is None:
        o = _like(q, stream)
    return _fwd(desc, q, q_chunk, cache, k, v, n_frames, o, 0, lse, stream)


def tm_sparse_causal_attn_fwd_f32out(desc: tm_attn_desc, q, q_chunk: int,
                                     cache: KVCache | None = None, k=None, v=None,
                                     n_frames: int = 0, o=None, lse=None, stream=None):
    """The same attention with an fp32 output (``o`` allocated as fp32 like q
    if not given); returns ``o``."""
    if o is None:
        o = _new(q.shape, torch.float32, q.device, stream)
    return _fwd(desc, q, q_chunk, cache, k, v, n_frames, o, 1, lse, stream)


def make_audio_desc(batch, heads, head_dim, tokens_per_frame, audio_per_frame, audio_frames,
                    streams=1, half_window=2, dtype="bf16", softmax_scale=0.0) -> tm_audio_desc:
    dtype = _dtype(dtype)
    return tm_audio_desc(batch, heads, head_dim, tokens_per_frame, audio_per_frame, audio_frames,
                         streams, half_window, dtype, softmax_scale)


def tm_audio_cross_attn_fwd(desc: tm_audio_desc, q, first_frame: int, ak, av, face, o=None,
                            n_tok: int | None = None, stream=None):
    """Audio cross-attention of the query rows ``q`` ([B, n_tok, H, D], row i
    in latent frame first_frame + i // T) over the audio keys/values ``ak``,
    ``av`` ([B, M, F_a * A, H, D]) with int32 face ids ``face`` ([B, n_tok]);
    returns ``o`` (allocated like q if not given)."""
    if n_tok is None:
        n_tok = q.shape[1]
    if o is None:
        o = _like(q, stream)
    _check(lib().tm_audio_cross_attn_fwd(ctypes.byref(desc), _ptr(q), first_frame, n_tok, _ptr(ak),
                                         _ptr(av), _ptr(face), _ptr(o), _stream(stream)))
    return o


def tm_audio_cross_attn_fwd_f32out(desc: tm_audio_desc, q, first_frame: int, ak, av, face,
                                   o=None, n_tok: int | None = None, stream=None):
    """The audio cross-attention with an fp32 output; returns ``o``."""
    if n_tok is None:
        n_tok = q.shape[1]
    if o is None:
        o = _new(q.shape, torch.float32, q.device, stream)
    _check(lib().tm_audio_cross_attn_fwd_f32out(ctypes.byref(desc), _ptr(q), first_frame, n_tok,
                                                _ptr(ak), _ptr(av), _ptr(face), _ptr(o),
                                                _stream(stream)))
    return o


def tm_sparse_causal_attn_bwd(desc: tm_attn_desc, n_frames: int, q, k, v, o, lse, dout, delta=None,
                              dq=None, dk=None, dv=None, stream=None):
    """Gradients (dq, dk, dv) of the full-sequence sparse causal attention;
    ``delta`` is an fp32 [B, H, L] workspace (allocated if not given). Where the
    sizes leave the GPU idle, the sums are shared out through a workspace of
    torch's allocator; calls that can have none (under capture, on another stream
    than the current one, with plain addresses) order them otherwise, as
    ``tm_sparse_causal_attn_bwd_noalloc`` does."""
    if delta is None:
        delta = _like(lse, stream)
    dq = _like(q, stream) if dq is None else dq
    dk = _like(k, stream) if dk is None else dk
    dv = _like(v, stream) if dv is None else dv
    d = ctypes.byref(desc)
    ptrs = [_ptr(t) for t in (q, k, v, o, lse, dout, delta, dq, dk, dv)]
    stream = _stream(stream)
    n = lib().tm_sparse_causal_attn_bwd_workspace(d, n_frames)
    ws = _workspace(n, q, stream)
    _check(lib().tm_sparse_causal_attn_bwd_ws(d, n_frames, *ptrs, _ptr(ws), n, stream))
    return dq, dk, dv


def tm_sparse_causal_attn_bwd_noalloc(desc: tm_attn_desc, n_frames: int, q, k, v, o, lse, dout,
                                      dq, dk, dv, stream=None):
    """The backward with the library's device-global workspace: the caller
    passes every output (nothing is allocated); returns (dq, dk, dv)."""
    _check(lib().tm_sparse_causal_attn_bwd_noalloc(ctypes.byref(desc), n_frames, _ptr(q), _ptr(k),
                                                   _ptr(v), _ptr(o), _ptr(lse), _ptr(dout),
                                                   _ptr(dq), _ptr(dk), _ptr(dv), _stream(stream)))
    return dq, dk, dv


def _expect(name, t, shape, dtype):
    """A tensor argument of the rotary and 8-bit-cache calls: the library sees
    addresses only, and torch's allocator puts many tensors into one allocation."""
    if t is not None and (t.shape != shape or t.dtype != dtype):
        raise TMError(TM_E_SHAPE, f"{name} is not {dtype} {list(shape)}")


def _rope_table_rows(desc):
    return lib().tm_rope3d_table_bytes(ctypes.byref(desc)) // 8


def make_rope_desc(head_dim, frames, grid_h, grid_w, pairs=None, theta=10000.0, split_half=False,
                   dtype="bf16") -> tm_rope_desc:
    """``pairs``: pairs turned by (frame, row, column); by default a third of
    them each for rows and columns and what is left for frames."""
    if pairs is None:
        third = head_dim // 2 // 3
        pairs = (head_dim // 2 - 2 * third, third, third)
    return tm_rope_desc(head_dim, frames, grid_h, grid_w, *pairs, int(bool(split_half)), _dtype(dtype), theta)


def tm_rope3d_table(desc: tm_rope_desc, table=None, device="cuda", stream=None):
    """(cos, sin) of every position and pair of the descriptor's axes, a flat
    fp32 tensor of pairs (allocated if not given)."""
    shape = (_rope_table_rows(desc), 2)
    if table is None:
        table = _new(shape, torch.float32, device, stream)
    _expect("table", table, shape, torch.float32)
    _check(lib().tm_rope3d_table(ctypes.byref(desc), _ptr(table), _stream(stream)))
    return table


def _rope(fn, desc, table, q, k, first_token, q_out, k_out, stream):
    # (one call per layer and token of a decoder: about 2 us are Python's, so nothing
    # is looked up twice, and no pointer of a tensor made here is checked)
    D, dtype, shape = desc.head_dim, _TORCH_DTYPE.get(desc.dtype), q.shape
    if len(shape) != 4 or shape[3] != D or q.dtype != dtype:
        raise TMError(TM_E_SHAPE, f"q is not {dtype} [batch, n_tok, heads, {D}]")
    B, n, H, _ = shape
    d = ctypes.byref(desc)
    if table is not None and (table.numel() * 4 != _lib.tm_rope3d_table_bytes(d) or table.dtype != torch.float32):
        raise TMError(TM_E_SHAPE, "table is not the descriptor's")
    if q_out is not None:
        _expect("q_out", q_out, shape, dtype)
    Hk, pk, pko = 0, None, None
    if k is not None:
        kshape = k.shape
        if len(kshape) != 4 or kshape[3] != D or k.dtype != dtype or kshape[0] != B or kshape[1] != n:
            raise TMError(TM_E_SHAPE, f"k is not {dtype} [{B}, {n}, kv_heads, {D}]")
        if k_out is not None:
            _expect("k_out", k_out, kshape, dtype)
        Hk, pk = kshape[2], _ptr(k)
        if k_out is None:
            k_out = _like(k, stream)
            pko = k_out.data_ptr()
        else:
            pko = _ptr(k_out)
    pq = _ptr(q)
    if q_out is None:
        q_out = _like(q, stream)
        pqo = q_out.data_ptr()
    else:
        pqo = _ptr(q_out)
    _check(fn(d, _ptr(table), B, n, first_token, pq, H, pk, Hk, pqo, pko, _stream(stream)))
    return q_out, k_out


def tm_rope3d_fwd(desc: tm_rope_desc, table, q, k=None, first_token: int = 0, q_out=None, k_out=None,
                  stream=None):
    """Rotate the rows of ``q`` ([B, n_tok, H, D]) and, if given, ``k`` ([B,
    n_tok, H_k, D]) by the latent frame, row and column of their token (row i is
    at position ``first_token`` + i); returns (q_out, k_out), allocated if not
    given."""
    return _rope(lib().tm_rope3d_fwd, desc, table, q, k, first_token, q_out, k_out, stream)


def tm_rope3d_bwd(desc: tm_rope_desc, table, dq_out, dk_out=None, first_token: int = 0, dq=None, dk=None,
                  stream=None):
    """Gradients (dq, dk) of ``tm_rope3d_fwd``'s inputs from those of its outputs."""
    return _rope(lib().tm_rope3d_bwd, desc, table, dq_out, dk_out, first_token, dq, dk, stream)


def tm_kv8_cache_tokens(desc: tm_attn_desc) -> int:
    return lib().tm_kv8_cache_tokens(ctypes.byref(desc))


def tm_kv8_cache_bytes(desc: tm_attn_desc, kv_heads: int) -> int:
    return lib().tm_kv8_cache_bytes(ctypes.byref(desc), kv_heads)


class KV8Cache:
    """A ``tm_kv8_cache`` handle together with the torch tensor that owns its
    pool (codes and scales). ``kv_heads``: key heads, the descriptor's heads by
    default."""

    def __init__(self, desc: tm_attn_desc, kv_heads: int | None = None, device="cuda", pool=None):
        self.desc = desc
        self.heads = desc.heads
        self.kv_heads = desc.heads if kv_heads is None else kv_heads
        self._batch, self._head_dim = desc.batch, desc.head_dim
        h = ctypes.c_void_p()
        if pool is None:
            n = tm_kv8_cache_bytes(desc, self.kv_heads)
            if n == 0:  # invalid: let the library say why
                _check(lib().tm_kv8_cache_create(ctypes.byref(desc), self.kv_heads, None, ctypes.byref(h)))
            pool = torch.empty(n, dtype=torch.uint8, device=device)
        elif pool.numel() * pool.element_size() < tm_kv8_cache_bytes(desc, self.kv_heads):
            raise TMError(TM_E_ARG, "pool is smaller than the cache")
        self.pool = pool
        _check(lib().tm_kv8_cache_create(ctypes.byref(desc), self.kv_heads, _ptr(pool), ctypes.byref(h)))
        self.handle = h
        self._at = ctypes.c_int32(), ctypes.c_int32()
        self._at_refs = tuple(ctypes.byref(x) for x in self._at)

    @property
    def capacity(self) -> int:
        return tm_kv8_cache_tokens(self.desc)

    def close(self):
        if getattr(self, "handle", None) is not None and _lib is not None:
            _lib.tm_kv8_cache_destroy(self.handle)
            self.handle = None

    __del__ = close

    def latest(self) -> int:
        return lib().tm_kv8_cache_latest(self.handle)

    def locate(self, chunk: int):
        # (one handle is not used by two threads at once)
        _check(lib().tm_kv8_cache_locate(self.handle, chunk, *self._at_refs))
        return self._at[0].value, self._at[1].value

    def reset(self):
        _check(lib().tm_kv8_cache_reset(self.handle))

    def rows(self, name, t, heads: int) -> int:
        """n of a tensor that has to be bf16 [batch, n, heads, head_dim] of the cache."""
        shape = t.shape
        if (len(shape) != 4 or shape[0] != self._batch or shape[2] != heads or shape[3] != self._head_dim
                or t.dtype != torch.bfloat16):
            raise TMError(TM_E_SHAPE, f"{name} is not bf16 [{self._batch}, n, {heads}, {self._head_dim}]")
        return shape[1]

    def kv_rows(self, k, v) -> int:
        n = self.rows("k", k, self.kv_heads)
        if self.rows("v", v, self.kv_heads) != n:
            raise TMError(TM_E_SHAPE, "k and v differ in tokens")
        return n


def tm_kv8_cache_create(desc: tm_attn_desc, kv_heads: int | None = None, device="cuda", pool=None) -> KV8Cache:
    return KV8Cache(desc, kv_heads, device, pool)


def tm_kv8_append(cache: KV8Cache, chunk: int, k, v, stream=None):
    """Quantise chunk ``chunk``'s K/V (bf16 ``[B, n_tok, kv_heads, D]``) into the cache."""
    n = cache.kv_rows(k, v)
    _check(lib().tm_kv8_append(cache.handle, chunk, _ptr(k), _ptr(v), n, _stream(stream)))


def tm_qkv8_produce(cache: KV8Cache, chunk: int, q, k, v, q_gain=None, k_gain=None, eps: float = 0.0,
                    rope: tm_rope_desc | None = None, table=None, first_token: int = 0, q_out=None,
                    stream=None):
    """RMS-normalise the chunk's q and k rows, rotate them if ``rope`` (with its
    ``table``) is given, and quantise k and v into the cache; returns ``q_out``
    (allocated like q if not given)."""
    n = cache.kv_rows(k, v)
    if cache.rows("q", q, cache.heads) != n:
        raise TMError(TM_E_SHAPE, "q and k differ in tokens")
    if q_gain is not None:
        _expect("q_gain", q_gain, (cache.heads, cache._head_dim), torch.float32)
    if k_gain is not None:
        _expect("k_gain", k_gain, (cache.kv_heads, cache._head_dim), torch.float32)
    d = None
    if rope is not None:
        d = ctypes.byref(rope)
        _expect("table", table, (_lib.tm_rope3d_table_bytes(d) // 8, 2), torch.float32)
    if q_out is not None:
        _expect("q_out", q_out, q.shape, torch.bfloat16)
    pq = _ptr(q)
    if q_out is None:
        q_out = _like(q, stream)
        pqo = q_out.data_ptr()
    else:
        pqo = _ptr(q_out)
    _check(_lib.tm_qkv8_produce(cache.handle, chunk, pq, _ptr(k), _ptr(v), _ptr(q_gain), _ptr(k_gain), eps, d,
                                _ptr(table), first_token, pqo, n, _stream(stream)))
    return q_out


def tm_kv8_read(cache: KV8Cache, chunk: int, dtype=torch.bfloat16, k_out=None, v_out=None, stream=None):
    """The keys and values that the cached chunk stands for, ``[B, n_tok,
    kv_heads, D]`` in bf16 or fp32 (allocated if not given)."""
    code = _dtype(dtype)
    dt = _TORCH_DTYPE[code]
    n, Hk, D = cache.locate(chunk)[1], cache.kv_heads, cache._head_dim
    shape = (cache._batch, n, Hk, D)
    if k_out is not None:
        _expect("k_out", k_out, shape, dt)
    if v_out is not None:
        _expect("v_out", v_out, shape, dt)
    if k_out is None:
        # (with its strides given: 0.3 us less than torch.empty)
        k_out = (torch.empty_strided(shape, (n * Hk * D, Hk * D, D, 1), dtype=dt, device=cache.pool.device)
                 if stream is None else _new(shape, dt, cache.pool.device, stream))
        pk = k_out.data_ptr()
    else:
        pk = _ptr(k_out)
    if v_out is None:
        v_out = _like(k_out, stream)
        pv = v_out.data_ptr()
    else:
        pv = _ptr(v_out)
    _check(_lib.tm_kv8_read(cache.handle, chunk, pk, pv, code == TM_F32, _stream(stream)))
    return k_out, v_out


def tm_kv8_attn_fwd(cache: KV8Cache, q, q_chunk: int, o=None, o_f32: bool = False, lse=None, stream=None):
    """Attention of the query rows ``q`` (bf16 ``[B, n_q, H, D]``, any number of
    rows of the latest chunk ``q_chunk``) over the 8-bit cache; returns ``o``
    (allocated like q, or as fp32, if not given). Rows that leave the GPU idle
    share their keys out through a workspace of torch's allocator; calls that
    can have none (under capture, on another stream than the current one) do
    not, and order the fp32 sums otherwise."""
    n_q = cache.rows("q", q, cache.heads)
    pq = _ptr(q)
    if o is None:
        o = _new(q.shape, torch.float32, q.device, stream) if o_f32 else _like(q, stream)
        po = o.data_ptr()
    else:
        _expect("o", o, q.shape, torch.float32 if o_f32 else torch.bfloat16)
        po = _ptr(o)
    pl = None
    if lse is not None:
        _expect("lse", lse, (cache._batch, cache.heads, n_q), torch.float32)
        pl = _ptr(lse)
    stream = _stream(stream)
    n = _lib.tm_kv8_attn_workspace(cache.handle, q_chunk, n_q)
    pw = None
    if n:
        ws = _workspace(n, q, stream)
        pw = None if ws is None else ws.data_ptr()
    _check(_lib.tm_kv8_attn_fwd(cache.handle, pq, q_chunk, n_q, po, o_f32, pl, pw, n, stream))
    return o


def _own_workspace(nbytes: int, given, like, stream: int):
    """The workspace that a backward call cannot do without: the caller's, or memory of torch's allocator
    (under capture, of the graph's pool), whose order is that of the current stream."""
    if nbytes == 0:
        return None
    if given is not None:
        if given.numel() * given.element_size() < nbytes:
            raise TMError(TM_E_ARG, f"workspace is smaller than {nbytes} bytes")
        return given
    if like.get_device() != torch._C._cuda_getDevice() or stream != _current_stream():
        raise TMError(TM_E_ARG, "on another stream or device than the current one, pass a workspace of "
                                f"{nbytes} bytes")
    return torch.empty(nbytes, dtype=torch.uint8, device=like.device)


def _rows(name, t, B, width, dtype) -> int:
    """n of a tensor that has to be [B, n, width] of the descriptor."""
    shape = t.shape
    if len(shape) != 3 or shape[0] != B or shape[2] != width or t.dtype != dtype:
        raise TMError(TM_E_SHAPE, f"{name} is not {dtype} [{B}, n, {width}]")
    return shape[1]


def _given(name, t, shape, dtype=torch.float32):
    """The address of a tensor that may be missing."""
    if t is None:
        return None
    if t.shape != shape or t.dtype != dtype:
        raise TMError(TM_E_SHAPE, f"{name} is not {dtype} {list(shape)}")
    return _ptr(t)


def _grad(name, t, of, stream):
    """The gradient of tensor ``of`` and its address: the caller's tensor, a new one like ``of`` if it is None,
    nothing if it is False or there is no ``of``."""
    if t is None:
        if of is None:
            return None, None
        t = _like(of, stream)
        return t, t.data_ptr()
    if t is False:
        return None, None
    if of is None:
        raise TMError(TM_E_ARG, f"{name} is the gradient of a tensor that is not there")
    _expect(name, t, of.shape, of.dtype)
    return t, _ptr(t)


def _formed(name, t, shape, dtype, like, stream):
    """A gradient that there always is, and its address: the caller's tensor, a new one if it is None, nothing if it
    is False."""
    if t is None:
        t = _new(shape, dtype, like.device, stream)
        return t, t.data_ptr()
    if t is False:
        return None, None
    return t, _given(name, t, shape, dtype)


def make_block_norm_desc(batch, width, pre="layer", post="none", dtype="bf16", stream_dtype="f32", eps=1e-6,
                         groups=1, group_tokens=0) -> tm_block_norm_desc:
    """``pre``, ``post``: "none", "layer" or "rms"; ``dtype`` of y and h, ``stream_dtype`` of x and r."""
    return tm_block_norm_desc(batch, width, _NORM_CODE.get(pre, pre), _NORM_CODE.get(post, post), _dtype(dtype),
                              _dtype(stream_dtype), groups, group_tokens, eps)


def tm_block_norm_fwd(desc: tm_block_norm_desc, x, y=None, gate=None, post_weight=None, pre_weight=None,
                      pre_bias=None, scale=None, shift=None, first_token: int = 0, r=None, h=None, stream=None):
    """r = x + gate * (post(y) * post_weight) and h = (pre(r) * pre_weight + pre_bias) * (1 + scale) + shift;
    returns (r, h), allocated if not given: r is None without y (x stands for it), h without pre."""
    B, E = desc.batch, desc.width
    act, st = _TORCH_DTYPE.get(desc.dtype), _TORCH_DTYPE.get(desc.stream_dtype)
    n = _rows("x", x, B, E, st)
    mod, vec, shape = (B, desc.groups, E), (E,), x.shape
    px, py, pr, ph = _ptr(x), None, None, None
    if y is not None:
        py = _given("y", y, shape, act)
        if r is None:
            r = torch.empty_like(x) if stream is None else _like(x, stream)
            pr = r.data_ptr()
        else:
            pr = _given("r", r, shape, st)
    elif r is not None:
        raise TMError(TM_E_ARG, "r goes with y")
    if desc.pre != TM_NORM_NONE:
        if h is None:
            h = torch.empty(shape, dtype=act, device=x.device) if stream is None else _new(shape, act, x.device, stream)
            ph = h.data_ptr()
        else:
            ph = _given("h", h, shape, act)
    elif h is not None:
        raise TMError(TM_E_ARG, "h goes with a norm before the block")
    _check(lib().tm_block_norm_fwd(
        ctypes.byref(desc), n, first_token, px, py, _given("gate", gate, mod), _given("post_weight", post_weight, vec),
        _given("pre_weight", pre_weight, vec), _given("pre_bias", pre_bias, vec), _given("scale", scale, mod),
        _given("shift", shift, mod), pr, ph, _stream(stream)))
    return r, h


_NO_SUMS = (None,) * 6


class BlockNormGrads(NamedTuple):
    """Gradients of ``tm_block_norm_fwd``'s inputs; None where the forward had no such input."""
    dx: torch.Tensor
    dy: torch.Tensor | None
    dgate: torch.Tensor | None
    dpost_weight: torch.Tensor | None
    dpre_weight: torch.Tensor | None
    dpre_bias: torch.Tensor | None
    dscale: torch.Tensor | None
    dshift: torch.Tensor | None


def tm_block_norm_bwd(desc: tm_block_norm_desc, r, dh=None, dr=None, y=None, gate=None, post_weight=None,
                      pre_weight=None, pre_bias=None, scale=None, shift=None, first_token: int = 0, dx=None, dy=None,
                      dgate=None, dpost_weight=None, dpre_weight=None, dpre_bias=None, dscale=None, dshift=None,
                      workspace=None, stream=None) -> BlockNormGrads:
    """Gradients of the block norm's inputs from dh and dr (None: r goes nowhere else), the forward's ``r`` (x
    without y; not read without a norm before the block) and its inputs. Each gradient is allocated if not given, and
    left out with False. ``workspace``: a tensor of ``tm_block_norm_bwd_workspace`` bytes (allocated if not given;
    needed on another stream than the current one)."""
    B, E = desc.batch, desc.width
    act, st = _TORCH_DTYPE.get(desc.dtype), _TORCH_DTYPE.get(desc.stream_dtype)
    has_pre = desc.pre != TM_NORM_NONE
    like = r if has_pre else dr
    if like is None:
        raise TMError(TM_E_ARG, "r is missing" if has_pre else "dr is missing without a norm before the block")
    n = _rows("r" if has_pre else "dr", like, B, E, st)
    shape, mod, vec = like.shape, (B, desc.groups, E), (E,)
    if (scale is None) != (shift is None):
        raise TMError(TM_E_ARG, "scale and shift: both or neither")
    ins = [_ptr(r) if has_pre else None, _given("dh", dh, shape, act), _given("dr", dr, shape, st),
           _given("y", y, shape, act), _given("gate", gate, mod), _given("post_weight", post_weight, vec),
           _given("pre_weight", pre_weight, vec), _given("pre_bias", pre_bias, vec), _given("scale", scale, mod)]
    _given("shift", shift, mod)
    if dx is False or dy is False:
        raise TMError(TM_E_ARG, "dx and dy are always formed")
    dx, pdx = _grad("dx", dx, like, stream)
    dy, pdy = _grad("dy", dy, y, stream)
    dgate, pdg = _grad("dgate", dgate, gate, stream)
    dpost_weight, pdp = _grad("dpost_weight", dpost_weight, post_weight, stream)
    dpre_weight, pdw = _grad("dpre_weight", dpre_weight, pre_weight, stream)
    dpre_bias, pdb = _grad("dpre_bias", dpre_bias, pre_bias, stream)
    dscale, pdc = _grad("dscale", dscale, scale, stream)
    dshift, pdh = _grad("dshift", dshift, scale, stream)
    d, stream = ctypes.byref(desc), _stream(stream)
    L = lib()
    nbytes, ws = 0, None
    if (pdg, pdp, pdw, pdb, pdc, pdh) != _NO_SUMS:
        nbytes = L.tm_block_norm_bwd_workspace(d, n, first_token)
        ws = _own_workspace(nbytes, workspace, like, stream)
    _check(L.tm_block_norm_bwd(d, n, first_token, *ins, pdx, pdy, pdg, pdp, pdw, pdb, pdc, pdh, _ptr(ws), nbytes,
                               stream))
    return BlockNormGrads(dx, dy, dgate, dpost_weight, dpre_weight, dpre_bias, dscale, dshift)


def make_linear_desc(batch, in_width, out_width, act="none", out_dtype="bf16", groups=1,
                     group_tokens=0) -> tm_linear_desc:
    """``act``: "none", "gelu" (its tanh form) or "silu"."""
    return tm_linear_desc(batch, in_width, out_width, _ACT_CODE.get(act, act), _dtype(out_dtype), groups,
                          group_tokens)


def tm_linear_fwd(desc: tm_linear_desc, x, weight, bias=None, gate=None, residual=None, first_token: int = 0, o=None,
                  pre=None, workspace=None, stream=None):
    """o = residual + gate * act(x W^T + bias) of bf16 ``x`` [B, n_tok, K] and ``weight`` [N, K]; returns ``o``
    (allocated if not given). ``pre`` (bf16 [B, n_tok, N]), if given, gets x W^T + bias for the backward pass.
    Sizes that leave CUs idle share their sums out through ``workspace`` (a tensor of ``tm_linear_fwd_workspace``
    bytes) or memory of torch's allocator; calls that have neither (under capture, on another stream than the
    current one) order the fp32 sums otherwise."""
    B, K, N = desc.batch, desc.in_width, desc.out_width
    out = _TORCH_DTYPE.get(desc.out_dtype)
    n = _rows("x", x, B, K, torch.bfloat16)
    shape = (B, n, N)
    px, pw = _ptr(x), _given("weight", weight, (N, K), torch.bfloat16)
    if o is None:
        o = torch.empty(shape, dtype=out, device=x.device) if stream is None else _new(shape, out, x.device, stream)
        po = o.data_ptr()
    else:
        po = _given("o", o, shape, out)
    pb, pg = _given("bias", bias, (N,)), _given("gate", gate, (B, desc.groups, N))
    pr, pp = _given("residual", residual, shape, out), _given("pre", pre, shape, torch.bfloat16)
    d, stream = ctypes.byref(desc), _stream(stream)
    L = lib()
    nbytes, ws = L.tm_linear_fwd_workspace(d, n), None
    if nbytes:
        if workspace is None:
            ws = _workspace(nbytes, x, stream)
        elif workspace.numel() * workspace.element_size() < nbytes:
            raise TMError(TM_E_ARG, f"workspace is smaller than {nbytes} bytes")
        else:
            ws = workspace
    _check(L.tm_linear_fwd(d, n, first_token, px, pw, pb, pg, pr, pp, po, _ptr(ws), nbytes, stream))
    return o


class LinearGrads(NamedTuple):
    """Gradients of ``tm_linear_fwd``'s inputs; None where one is not wanted, and dgate where the forward had no gate.
    (dbias is formed unless it is False: the backward does not see the bias. The residual's is the output's.)"""
    dx: torch.Tensor | None
    dweight: torch.Tensor | None
    dbias: torch.Tensor | None
    dgate: torch.Tensor | None


def tm_linear_bwd(desc: tm_linear_desc, x, weight, dout, gate=None, pre=None, first_token: int = 0, dx=None,
                  dweight=None, dbias=None, dgate=None, workspace=None, stream=None) -> LinearGrads:
    """Gradients from that of the output, ``dout``. ``pre``: the forward's (not needed without activation and
    gate; nor ``x`` without dweight and ``weight`` without dx). Each gradient is allocated if not given, and left out
    with False (the bias' for a layer without).
    ``workspace``: a tensor of ``tm_linear_bwd_workspace`` bytes (allocated if not given; needed on another
    stream than the current one)."""
    B, K, N = desc.batch, desc.in_width, desc.out_width
    n = _rows("dout", dout, B, N, _TORCH_DTYPE.get(desc.out_dtype))
    px, pw = _given("x", x, (B, n, K), _BF16), _given("weight", weight, (N, K), _BF16)
    pd, pg, pp = _ptr(dout), _given("gate", gate, (B, desc.groups, N)), _given("pre", pre, (B, n, N), _BF16)
    dx, pdx = _formed("dx", dx, (B, n, K), _BF16, dout, stream)
    dweight, pdw = _formed("dweight", dweight, (N, K), _BF16, dout, stream)
    dbias, pdb = _formed("dbias", dbias, (N,), torch.float32, dout, stream)
    dgate, pdg = _grad("dgate", dgate, gate, stream)
    d, stream = ctypes.byref(desc), _stream(stream)
    nbytes = lib().tm_linear_bwd_workspace(d, n, first_token)
    ws = _own_workspace(nbytes, workspace, dout, stream)
    _check(lib().tm_linear_bwd(d, n, first_token, px, pw, pd, pg, pp, pdx, pdw, pdb, pdg, _ptr(ws), nbytes, stream))
    return LinearGrads(dx, dweight, dbias, dgate)
