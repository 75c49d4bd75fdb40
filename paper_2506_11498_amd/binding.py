"""Thin ctypes binding of liblrsa.so: argument marshalling only.

Every step of the path (score, select, attention forward and backward) runs in the HIP
kernels behind the C ABI declared in include/lrsa.h; torch is used here for device memory
and the current stream, nothing else.  There is no CPU fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblrsa.so")

LRSA_F32, LRSA_BF16 = 0, 1
IMPL_AUTO, IMPL_GENERIC, IMPL_COMPACT = 0, 1, 2
WS_SCORE, WS_SELECT, WS_ATTN_FWD, WS_ATTN_BWD, WS_DECODE_ATTN = 0, 1, 2, 3, 4

EXPORTS = ("lrsa_abi_version", "lrsa_last_error", "lrsa_num_scored_chunks", "lrsa_score_route", "lrsa_attn_route", "lrsa_score_poll_limit", "lrsa_workspace_bytes",
           "lrsa_score", "lrsa_select", "lrsa_score_select", "lrsa_check_idx", "lrsa_attn_fwd", "lrsa_attn_bwd",
           "lrsa_cache_compress", "lrsa_cache_compress_ws", "lrsa_cache_compress_ws_bytes", "lrsa_decode_attn", "lrsa_decode_attn_static",
           "lrsa_fill_workspace_bytes", "lrsa_attn_bwd_parts", "lrsa_attn_plan", "lrsa_attn_fwd_fill", "lrsa_attn_bwd_fill", "lrsa_attn_bwd_finish",
           "lrsa_decode_attn_acc", "lrsa_decode_attn_acc_ws_bytes", "lrsa_cache_evict", "lrsa_cache_evict_ws_bytes",
           "lrsa_cache_append_quant", "lrsa_cache_read_quant", "lrsa_decode_attn_quant", "lrsa_decode_attn_quant_ws_bytes", "lrsa_cache_evict_quant",
           "lrsa_timing_enable", "lrsa_timing_count", "lrsa_timing_read")


class LrsaParams(ctypes.Structure):
    """Mirror of lrsa_params in include/lrsa.h."""
    _fields_ = [
        ("batch", ctypes.c_int32), ("heads_q", ctypes.c_int32), ("heads_kv", ctypes.c_int32),
        ("seq", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("sink", ctypes.c_int32), ("lag", ctypes.c_int32), ("topk", ctypes.c_int32),
        ("std_ddof", ctypes.c_int32), ("local_prev", ctypes.c_int32),
        ("softmax_scale", ctypes.c_float), ("dtype", ctypes.c_int32), ("impl", ctypes.c_int32),
        ("q_stride", ctypes.c_int64 * 3), ("kv_stride", ctypes.c_int64 * 3),
    ]


class LrsaQuantCache(ctypes.Structure):
    """Mirror of lrsa_quant_cache in include/lrsa.h."""
    _fields_ = [("format", ctypes.c_int32), ("block", ctypes.c_int32), ("stride", ctypes.c_int64 * 3),
                ("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("K_scale", ctypes.c_void_p), ("V_scale", ctypes.c_void_p)]


class LrsaError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"liblrsa error {code}: {msg}")
        self.code = code


_lib = None


def lib() -> ctypes.CDLL:
    """Load liblrsa.so (built in-tree by paper_2506_11498_amd.build); fail loudly if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is not built; run `python -m paper_2506_11498_amd.build` "
                                    "(or __graft_entry__.build()).  There is no fallback path.")
        L = ctypes.CDLL(LIB_PATH)
        L.lrsa_last_error.restype = ctypes.c_char_p
        L.lrsa_workspace_bytes.restype = ctypes.c_size_t
        L.lrsa_workspace_bytes.argtypes = [ctypes.c_void_p, ctypes.c_int]
        L.lrsa_num_scored_chunks.argtypes = [ctypes.c_void_p]
        L.lrsa_score_route.argtypes = [ctypes.c_void_p]
        L.lrsa_attn_route.argtypes = [ctypes.c_void_p]
        L.lrsa_score_poll_limit.argtypes = [ctypes.c_int]
        L.lrsa_score_poll_limit.restype = ctypes.c_int
        vp, sz = ctypes.c_void_p, ctypes.c_size_t
        L.lrsa_score.argtypes = [vp, vp, vp, vp, vp, sz, vp]
        L.lrsa_select.argtypes = [vp, vp, vp, vp, sz, vp]
        L.lrsa_score_select.argtypes = [vp, vp, vp, vp, vp, vp, sz, vp]
        L.lrsa_check_idx.argtypes = [vp, vp, vp, vp]
        L.lrsa_cache_compress.argtypes = [vp, vp, vp, vp, ctypes.c_int32, ctypes.c_int32, vp, vp, vp]
        L.lrsa_cache_compress_ws_bytes.restype = ctypes.c_size_t
        L.lrsa_cache_compress_ws_bytes.argtypes = [vp, ctypes.c_int32, ctypes.c_int32]
        L.lrsa_cache_compress_ws.argtypes = [vp, vp, vp, vp, ctypes.c_int32, ctypes.c_int32, vp, vp, vp, sz, vp]
        L.lrsa_decode_attn.argtypes = [vp, vp, vp, vp, ctypes.c_int32, vp, vp, vp, sz, vp]
        L.lrsa_decode_attn_static.argtypes = [vp, vp, vp, vp, ctypes.c_int32, vp, vp, vp]
        i32 = ctypes.c_int32
        L.lrsa_fill_workspace_bytes.restype = ctypes.c_size_t
        L.lrsa_fill_workspace_bytes.argtypes = [vp, i32, i32, ctypes.c_int]
        L.lrsa_attn_bwd_parts.argtypes = [vp, i32, i32, vp, vp]
        L.lrsa_attn_plan.argtypes = [vp, i32, i32, sz, vp]
        L.lrsa_attn_fwd_fill.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.lrsa_attn_bwd_fill.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.lrsa_attn_bwd_finish.argtypes = [vp, vp, vp, vp, vp, vp]
        L.lrsa_attn_fwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.lrsa_attn_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        f32 = ctypes.c_float
        L.lrsa_decode_attn_acc_ws_bytes.restype = sz
        L.lrsa_decode_attn_acc_ws_bytes.argtypes = [vp, i32]
        L.lrsa_decode_attn_acc.argtypes = [vp, vp, vp, vp, i32, vp, vp, f32, vp, vp, vp, sz, vp]
        L.lrsa_cache_evict_ws_bytes.restype = sz
        L.lrsa_cache_evict_ws_bytes.argtypes = [vp, i32, i32]
        L.lrsa_cache_evict.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
        L.lrsa_cache_append_quant.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp]
        L.lrsa_cache_read_quant.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp]
        L.lrsa_decode_attn_quant_ws_bytes.restype = sz
        L.lrsa_decode_attn_quant_ws_bytes.argtypes = [vp, i32, i32, ctypes.c_int]
        L.lrsa_decode_attn_quant.argtypes = [vp, vp, vp, i32, vp, i32, vp, vp, f32, vp, vp, vp, sz, vp]
        L.lrsa_cache_evict_quant.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        _lib = L
    return _lib


def _check(rc: int):
    if rc < 0:
        raise LrsaError(rc, lib().lrsa_last_error().decode())
    return rc


def make_params(q_shape, kv_shape, q_stride, kv_stride, *, sink: int, lag: int, topk: int, dtype,
                std_ddof: int = 1, local_prev: int = 1, softmax_scale: float = 0.0,
                impl: int = IMPL_AUTO) -> LrsaParams:
    """Build lrsa_params from [B,H,n,d] shapes and element strides (the last stride must be 1)."""
    B, Hq, n, d = q_shape
    if q_stride[3] != 1 or kv_stride[3] != 1:
        raise ValueError("the channel stride must be 1")
    p = LrsaParams()
    p.batch, p.heads_q, p.heads_kv, p.seq, p.head_dim = B, Hq, kv_shape[1], n, d
    p.sink, p.lag, p.topk, p.std_ddof, p.local_prev = sink, lag, topk, std_ddof, local_prev
    p.softmax_scale = softmax_scale
    p.dtype = LRSA_F32 if dtype == torch.float32 else LRSA_BF16 if dtype == torch.bfloat16 else -1
    p.impl = impl
    for i in range(3):
        p.q_stride[i] = q_stride[i]
        p.kv_stride[i] = kv_stride[i]
    return p


def params_for(Q: torch.Tensor, K: torch.Tensor, **kw) -> LrsaParams:
    return make_params(tuple(Q.shape), tuple(K.shape), Q.stride(), K.stride(), dtype=Q.dtype, **kw)


def num_scored_chunks(p: LrsaParams) -> int:
    return _check(lib().lrsa_num_scored_chunks(ctypes.byref(p)))


def score_route(p: LrsaParams) -> int:
    """Which kernels score these params: 0 none, 1 one workgroup per chunk, 2 sliced, 3 one read (rows kept in
    registers), 4 long chunks."""
    return _check(lib().lrsa_score_route(ctypes.byref(p)))


def attn_route(p: LrsaParams) -> int:
    """Which attention kernels these params get: 0 plain fp32-arithmetic, 1 fp32 matrix kernels, 2 bf16 MFMA."""
    return _check(lib().lrsa_attn_route(ctypes.byref(p)))


def score_poll_limit(polls: int) -> int:
    """Sets how often a one-read scoring workgroup polls for its hint words (negative: query only); returns the
    previous value.  Results do not depend on it."""
    return int(lib().lrsa_score_poll_limit(int(polls)))


def workspace_bytes(p: LrsaParams, which: int) -> int:
    return int(lib().lrsa_workspace_bytes(ctypes.byref(p), which))


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()   # argtypes make a pointer of it


# The handle of the current device's current stream, as torch.cuda.current_stream().cuda_stream gives it.  That builds a Stream object,
# 3 of the 12 us that a call of lrsa_decode_attn took on the host (11.9 us a call, 7.8 on the GPU), hence the raw handle where torch has it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    if _raw_stream is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


_TORCH_DTYPE = {LRSA_F32: torch.float32, LRSA_BF16: torch.bfloat16}


def _expect(name: str, t: Optional[torch.Tensor], shape, stride, dtype, device) -> None:
    """The C ABI describes Q, O, dO, dQ by ONE stride triple and K, V, dK, dV by another, and takes score, idx,
    lse as contiguous: a tensor that differs would be read or written at wrong addresses, so it is refused."""
    if t is None:
        return
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype != dtype:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {dtype}")
    if t.device != device:
        raise ValueError(f"{name}: on {t.device}, expected {device}")
    if stride is None:
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    else:
        for dim, (have, want) in enumerate(zip(t.stride(), stride)):
            if t.shape[dim] > 1 and have != want:
                raise ValueError(f"{name}: stride {tuple(t.stride())}, the params describe {tuple(stride)}")


def _expect_q(p: LrsaParams, device, **tensors) -> None:
    shape = (p.batch, p.heads_q, p.seq, p.head_dim)
    for name, t in tensors.items():
        _expect(name, t, shape, (*p.q_stride, 1), _TORCH_DTYPE.get(p.dtype), device)


def _expect_kv(p: LrsaParams, device, **tensors) -> None:
    shape = (p.batch, p.heads_kv, p.seq, p.head_dim)
    for name, t in tensors.items():
        _expect(name, t, shape, (*p.kv_stride, 1), _TORCH_DTYPE.get(p.dtype), device)


def _workspace(p: LrsaParams, which: int, device, ws: Optional[torch.Tensor]) -> Tuple[Optional[torch.Tensor], int]:
    need = workspace_bytes(p, which)
    if need == 0:
        return None, 0
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=device)
    return ws, ws.numel() * ws.element_size()


def lrsa_score(p: LrsaParams, K: torch.Tensor, V: torch.Tensor, score: Optional[torch.Tensor] = None,
               ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """LagKV scores [B, Hkv, Ns, L] fp32 (Eq. 4-8)."""
    Ns = num_scored_chunks(p)
    if score is None:
        score = torch.empty((p.batch, p.heads_kv, Ns, p.lag), dtype=torch.float32, device=K.device)
    _expect_kv(p, K.device, K=K, V=V)
    _expect("score", score, (p.batch, p.heads_kv, Ns, p.lag), None, torch.float32, K.device)
    ws, nb = _workspace(p, WS_SCORE, K.device, ws)
    _check(lib().lrsa_score(ctypes.byref(p), _ptr(K), _ptr(V), _ptr(score), _ptr(ws), nb, _stream()))
    return score


def lrsa_select(p: LrsaParams, score: torch.Tensor, idx: Optional[torch.Tensor] = None,
                ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Top-K positions per (batch, KV head, chunk): int32 [B, Hkv, Ns, K], ascending."""
    Ns = num_scored_chunks(p)
    if idx is None:
        idx = torch.empty((p.batch, p.heads_kv, Ns, p.topk), dtype=torch.int32, device=score.device)
    _expect("score", score, (p.batch, p.heads_kv, Ns, p.lag), None, torch.float32, score.device)
    _expect("idx", idx, (p.batch, p.heads_kv, Ns, p.topk), None, torch.int32, score.device)
    ws, nb = _workspace(p, WS_SELECT, score.device, ws)
    _check(lib().lrsa_select(ctypes.byref(p), _ptr(score), _ptr(idx), _ptr(ws), nb, _stream()))
    return idx


def lrsa_check_idx(p: LrsaParams, idx: Optional[torch.Tensor], bad_rows: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Number of rows of idx that are not K ascending positions of their chunk, as a device int32 tensor of one
    element (0 for a valid idx).  Enqueued like every call: `.item()` on the result synchronises."""
    Ns = num_scored_chunks(p)
    device = idx.device if idx is not None else torch.device("cuda", torch.cuda.current_device())
    if idx is not None:
        _expect("idx", idx, (p.batch, p.heads_kv, Ns, p.topk), None, torch.int32, device)
    if bad_rows is None:
        bad_rows = torch.empty(1, dtype=torch.int32, device=device)
    _expect("bad_rows", bad_rows, (1,), None, torch.int32, device)
    _check(lib().lrsa_check_idx(ctypes.byref(p), _ptr(idx), _ptr(bad_rows), _stream()))
    return bad_rows


def lrsa_score_select(p: LrsaParams, K: torch.Tensor, V: torch.Tensor, score: Optional[torch.Tensor] = None,
                      idx: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """lrsa_score and lrsa_select in one call (the selection is taken by the kernel that finishes the scores):
    (score, idx)."""
    Ns = num_scored_chunks(p)
    if score is None:
        score = torch.empty((p.batch, p.heads_kv, Ns, p.lag), dtype=torch.float32, device=K.device)
    if idx is None:
        idx = torch.empty((p.batch, p.heads_kv, Ns, p.topk), dtype=torch.int32, device=K.device)
    _expect_kv(p, K.device, K=K, V=V)
    _expect("score", score, (p.batch, p.heads_kv, Ns, p.lag), None, torch.float32, K.device)
    _expect("idx", idx, (p.batch, p.heads_kv, Ns, p.topk), None, torch.int32, K.device)
    ws, nb = _workspace(p, WS_SCORE, K.device, ws)
    _check(lib().lrsa_score_select(ctypes.byref(p), _ptr(K), _ptr(V), _ptr(score), _ptr(idx), _ptr(ws), nb, _stream()))
    return score, idx


def cache_compress_ws_bytes(p: LrsaParams, length: int, done: int) -> int:
    """Workspace of lrsa_cache_compress for these counts; 0 where nothing moves or a single step is the faster one without."""
    return int(lib().lrsa_cache_compress_ws_bytes(ctypes.byref(p), int(length), int(done)))


def lrsa_cache_compress(p: LrsaParams, Kc: torch.Tensor, Vc: torch.Tensor, pos: Optional[torch.Tensor],
                        length: int, done: int, ws: Optional[torch.Tensor] = None):
    """Inference-time cache: compress (in place) while the uncompressed tail holds 2*lag rows.
    Kc, Vc: [B, Hkv, cap, d] with cap = p.seq; pos: int32 [B, Hkv, cap] or None.  Returns (length, done).
    ws: cache_compress_ws_bytes() bytes.  Without one, a workspace is allocated for the call; under graph capture (where nothing
    would hold it until the replays) and where there is no memory for it, the same steps run one by one without."""
    L, pp, new_len, new_done = lib(), ctypes.byref(p), ctypes.c_int32(0), ctypes.c_int32(0)
    length, done = int(length), int(done)
    need = L.lrsa_cache_compress_ws_bytes(pp, length, done) if Kc is not None else 0
    if need and ws is None and not torch.cuda.is_current_stream_capturing():
        try:
            ws = torch.empty(need, dtype=torch.uint8, device=Kc.device)
        except torch.OutOfMemoryError:
            pass
    args = (pp, _ptr(Kc), _ptr(Vc), _ptr(pos), length, done, ctypes.byref(new_len), ctypes.byref(new_done))
    if need and ws is None:
        _check(L.lrsa_cache_compress(*args, _stream()))
    else:
        _check(L.lrsa_cache_compress_ws(*args, _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(), _stream()))
    return new_len.value, new_done.value


def lrsa_decode_attn(p: LrsaParams, q: torch.Tensor, Kc: torch.Tensor, Vc: torch.Tensor, length: int,
                     O: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                     ws: Optional[torch.Tensor] = None):
    """Single-query attention over cache rows [0, length): q, O [B, Hq, d]; returns (O, lse [B, Hq] fp32)."""
    if O is None:
        O = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((p.batch, p.heads_q), dtype=torch.float32, device=q.device)
    ws, nb = _workspace(p, WS_DECODE_ATTN, q.device, ws)
    _check(lib().lrsa_decode_attn(ctypes.byref(p), _ptr(q), _ptr(Kc), _ptr(Vc), int(length), _ptr(O), _ptr(lse),
                                  _ptr(ws), nb, _stream()))
    return O, lse


def lrsa_decode_attn_static(p: LrsaParams, q: torch.Tensor, Kc: torch.Tensor, Vc: torch.Tensor, length: int,
                            O: torch.Tensor, lse: Optional[torch.Tensor]):
    """lrsa_decode_attn without a workspace (the library's built-in scratch array); O and lse are the caller's."""
    _check(lib().lrsa_decode_attn_static(ctypes.byref(p), _ptr(q), _ptr(Kc), _ptr(Vc), int(length), _ptr(O), _ptr(lse),
                                         _stream()))
    return O, lse


# ---- accumulated weights, eviction, the cache in 8 bits
# A single token's call takes the GPU 10 us, as long as the checks of its dozen tensors took on the host when they were written like those
# above (lrsa_cache_evict 21.8 us a call).  So here the params are read in one go, and a tensor that fits is recognised by four
# comparisons; only one that does not goes through _expect, which says why.
_PARAMS = struct.Struct("@10if2i6q")


def _read(p: LrsaParams):
    """(batch, heads_q, heads_kv, seq, head_dim), torch dtype, (strides of K and V rows)"""
    f = _PARAMS.unpack_from(p)
    return f[:5], _TORCH_DTYPE.get(f[11]), f[16:19]


def _here(t: torch.Tensor) -> int:
    """The library launches on the current device's current stream: tensors that live elsewhere are refused."""
    i = t.get_device()
    if i < 0 or i != torch.cuda.current_device():
        raise ValueError(f"tensors on {t.device}, expected the current CUDA device")
    return i


def _stream_of(index: int):
    return _stream() if _raw_stream is None else _raw_stream(index)


def _flat(name: str, t: Optional[torch.Tensor], shape, dtype, index: int) -> Optional[int]:
    """The address of a contiguous tensor of that shape."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index or not t.is_contiguous():
        _expect(name, t, shape, None, dtype, torch.device("cuda", index))
    return t.data_ptr()


def _rows(name: str, t: Optional[torch.Tensor], shape, stride, dtype, index: int) -> Optional[int]:
    """The address of a tensor of that shape and those strides."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index or t.stride() != stride:
        _expect(name, t, shape, stride, dtype, torch.device("cuda", index))
    return t.data_ptr()


def _own_ws(need: int, index: int) -> torch.Tensor:
    return torch.empty(need, dtype=torch.uint8, device=torch.device("cuda", index))


def _ws_at(ws: torch.Tensor, index: int) -> int:
    if ws.get_device() != index or not ws.is_contiguous():
        raise ValueError(f"ws must be contiguous and on cuda:{index}")
    return ws.data_ptr()


def decode_attn_acc_ws_bytes(p: LrsaParams, length: int) -> int:
    return int(lib().lrsa_decode_attn_acc_ws_bytes(ctypes.byref(p), int(length)))


def lrsa_decode_attn_acc(p: LrsaParams, q: torch.Tensor, Kc: torch.Tensor, Vc: torch.Tensor, length: int, acc_in: Optional[torch.Tensor],
                         acc_out: torch.Tensor, decay: float = 1.0, O: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                         ws: Optional[torch.Tensor] = None):
    """lrsa_decode_attn that also writes acc_out = decay * acc_in + the weight that every cache row received, summed over the heads of
    its group: acc [B, Hkv, cap] fp32, acc_in None for zeros, both may be the same tensor.  Returns (O, lse, acc_out)."""
    index, dev, f32 = _here(q), q.device, torch.float32
    (B, Hq, Hkv, cap, d), dt, ks = _read(p)
    if O is None:
        O = torch.empty((B, Hq, d), dtype=q.dtype, device=dev)
    if lse is None:
        lse = torch.empty((B, Hq), dtype=f32, device=dev)
    one, kv, st, acc = (B, Hq, d), (B, Hkv, cap, d), (*ks, 1), (B, Hkv, cap)
    args = (_flat("q", q, one, dt, index), _rows("Kc", Kc, kv, st, dt, index), _rows("Vc", Vc, kv, st, dt, index), length,
            _flat("acc_in", acc_in, acc, f32, index), _flat("acc_out", acc_out, acc, f32, index), decay, _flat("O", O, one, dt, index),
            _flat("lse", lse, (B, Hq), f32, index))
    if ws is None:
        ws = _own_ws(decode_attn_acc_ws_bytes(p, length), index)
    _check(lib().lrsa_decode_attn_acc(ctypes.byref(p), *args, _ws_at(ws, index), ws.nbytes, _stream_of(index)))
    return O, lse, acc_out


def cache_evict_ws_bytes(p: LrsaParams, length: int, budget: int) -> int:
    """Workspace of lrsa_cache_evict, and of lrsa_cache_evict_quant with its max_len as the length."""
    return int(lib().lrsa_cache_evict_ws_bytes(ctypes.byref(p), int(length), int(budget)))


def lrsa_cache_evict(p: LrsaParams, Kc: torch.Tensor, Vc: torch.Tensor, pos: Optional[torch.Tensor], acc: torch.Tensor, length: int, budget: int,
                     recent: int, Ko: torch.Tensor, Vo: torch.Tensor, pos_o: Optional[torch.Tensor], acc_o: torch.Tensor,
                     ws: Optional[torch.Tensor] = None) -> int:
    """The first p.sink rows, the last `recent` and those of the others with the largest acc, `budget` in all, go to the cache Ko, Vo
    (with their positions and weights; weights behind them become zero).  Returns the new length."""
    index, dev, i32, f32 = _here(Kc), Kc.device, torch.int32, torch.float32
    (B, _, Hkv, cap, d), dt, ks = _read(p)
    kv, st, lst, new = (B, Hkv, cap, d), (*ks, 1), (B, Hkv, cap), ctypes.c_int32(0)
    args = (_rows("Kc", Kc, kv, st, dt, index), _rows("Vc", Vc, kv, st, dt, index), _flat("pos", pos, lst, i32, index), _flat("acc", acc, lst, f32, index),
            length, budget, recent, _rows("Ko", Ko, kv, st, dt, index), _rows("Vo", Vo, kv, st, dt, index), _flat("pos_o", pos_o, lst, i32, index),
            _flat("acc_o", acc_o, lst, f32, index))
    if ws is None:
        ws = _own_ws(cache_evict_ws_bytes(p, length, budget), index)
    _check(lib().lrsa_cache_evict(ctypes.byref(p), *args, ctypes.byref(new), _ws_at(ws, index), ws.nbytes, _stream_of(index)))
    return new.value


_QUANT_FORMATS = {torch.int8: 0, torch.float8_e4m3fn: 1}


class QuantCache:
    """The K and V of a cache in 8 bits: codes [B, Hkv, cap, d] (torch.int8 or torch.float8_e4m3fn, K and V by the same strides) and
    fp32 scales [B, Hkv, ceil(cap / block)] of blocks of 16, 32, 64 or 128 rows.  Holds the tensors and the struct that the library reads."""

    def __init__(self, K: torch.Tensor, V: torch.Tensor, K_scale: torch.Tensor, V_scale: torch.Tensor, block: int):
        if K.dtype not in _QUANT_FORMATS:
            raise ValueError(f"codes are torch.int8 or torch.float8_e4m3fn, not {K.dtype}")
        if K.dim() != 4 or K.stride(3) != 1:
            raise ValueError("codes are [B, Hkv, cap, d] with a channel stride of 1")
        if block not in (16, 32, 64, 128):
            raise ValueError(f"blocks of {block} rows are not built (16, 32, 64 and 128 are)")
        B, Hkv, cap, d = K.shape
        _expect("V", V, K.shape, K.stride(), K.dtype, K.device)
        for name, t in (("K_scale", K_scale), ("V_scale", V_scale)):
            _expect(name, t, (B, Hkv, -(-cap // block)), None, torch.float32, K.device)
        self._tensors = K, V, K_scale, V_scale          # the struct holds their addresses: they are not exchanged
        self.block, self.shape, self.device = block, (B, Hkv, cap, d), K.device
        # the stride of an axis of length 1 is whatever torch made it: any multiple of 16 serves
        st = [s if n > 1 else d for s, n in zip(K.stride()[:3], K.shape[:3])]
        self.struct = LrsaQuantCache(_QUANT_FORMATS[K.dtype], block, (ctypes.c_int64 * 3)(*st), *(t.data_ptr() for t in self._tensors))
        self.ref = ctypes.byref(self.struct)

    K, V, K_scale, V_scale = (property(lambda self, i=i: self._tensors[i]) for i in range(4))

    @classmethod
    def empty(cls, B: int, Hkv: int, cap: int, d: int, dtype=torch.int8, block: int = 64, device="cuda") -> "QuantCache":
        codes = [torch.zeros((B, Hkv, cap, d), dtype=torch.uint8, device=device).view(dtype) for _ in range(2)]
        return cls(*codes, *(torch.ones((B, Hkv, -(-cap // block)), dtype=torch.float32, device=device) for _ in range(2)), block)

    def _as(self, name: str, shape, device):
        """The reference that the library takes, of a cache that the params describe (its tensors were checked when it was made)."""
        if self.shape != shape:
            raise ValueError(f"{name}: codes {self.shape}, the params describe {shape}")
        if self.device != device:
            raise ValueError(f"{name}: on {self.device}, expected {device}")
        return self.ref


def lrsa_cache_append_quant(p: LrsaParams, cache: QuantCache, K: torch.Tensor, V: torch.Tensor, lens: torch.Tensor,
                            counts: Optional[torch.Tensor] = None) -> None:
    """Rows lens[b] .. of the cache become the first counts[b] (None: all) rows of K and V [B, Hkv, tokens, d], strides as p.kv_stride says;
    lens, counts: [B] int32 on the device, not changed."""
    index, dev, i32 = _here(K), K.device, torch.int32
    (B, _, Hkv, cap, d), dt, ks = _read(p)
    tokens = K.shape[2]
    kv, st = (B, Hkv, tokens, d), (*ks, 1)
    _check(lib().lrsa_cache_append_quant(ctypes.byref(p), cache._as("cache", (B, Hkv, cap, d), dev), _rows("K", K, kv, st, dt, index),
                                         _rows("V", V, kv, st, dt, index), tokens, _flat("lens", lens, (B,), i32, index),
                                         _flat("counts", counts, (B,), i32, index), _stream_of(index)))


def lrsa_cache_read_quant(p: LrsaParams, cache: QuantCache, lens: torch.Tensor, rows: int, first: Optional[torch.Tensor] = None,
                          K: Optional[torch.Tensor] = None, V: Optional[torch.Tensor] = None):
    """Rows first[b] (None: 0) .. + rows of every sequence as values [B, Hkv, rows, d], zero at and behind lens[b]; returns (K, V), by
    default of the strides that p.kv_stride gives (refused where they are made for fewer rows)."""
    index, dev, i32 = _here(lens), lens.device, torch.int32
    (B, _, Hkv, cap, d), dt, ks = _read(p)
    kv, st = (B, Hkv, rows, d), (*ks, 1)
    K, V = (torch.empty_strided(kv, st, dtype=dt, device=dev) if t is None else t for t in (K, V))
    _check(lib().lrsa_cache_read_quant(ctypes.byref(p), cache._as("cache", (B, Hkv, cap, d), dev), _flat("lens", lens, (B,), i32, index), rows,
                                       _flat("first", first, (B,), i32, index), _rows("K", K, kv, st, dt, index), _rows("V", V, kv, st, dt, index),
                                       _stream_of(index)))
    return K, V


def decode_attn_quant_ws_bytes(p: LrsaParams, tokens: int, max_len: int, with_acc: bool) -> int:
    return int(lib().lrsa_decode_attn_quant_ws_bytes(ctypes.byref(p), int(tokens), int(max_len), 1 if with_acc else 0))


def lrsa_decode_attn_quant(p: LrsaParams, q: torch.Tensor, cache: QuantCache, lens: torch.Tensor, max_len: int, acc_in: Optional[torch.Tensor] = None,
                           acc_out: Optional[torch.Tensor] = None, decay: float = 1.0, O: Optional[torch.Tensor] = None,
                           lse: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """Attention of the last tokens of every sequence over the cache: q, O [B, Hq, tokens, d] (or [B, Hq, d]: one token), lens [B] int32 on
    the device, none above max_len; token t sees the rows below lens[b] - tokens + 1 + t.  With acc_out, the rows' weights are added up
    as in lrsa_decode_attn_acc.  Returns (O, lse [B, Hq, tokens] fp32)."""
    index, dev, f32 = _here(q), q.device, torch.float32
    (B, Hq, Hkv, cap, d), dt, _ = _read(p)
    tokens = q.shape[2] if q.dim() == 4 else 1
    rows = (B, Hq, tokens) if q.dim() == 4 else (B, Hq)
    shape, acc = (*rows, d), (B, Hkv, cap)
    if O is None:
        O = torch.empty(shape, dtype=q.dtype, device=dev)
    if lse is None:
        lse = torch.empty(rows, dtype=f32, device=dev)
    args = (cache._as("cache", (B, Hkv, cap, d), dev), _flat("q", q, shape, dt, index), tokens, _flat("lens", lens, (B,), torch.int32, index), max_len,
            _flat("acc_in", acc_in, acc, f32, index), _flat("acc_out", acc_out, acc, f32, index), decay, _flat("O", O, shape, dt, index),
            _flat("lse", lse, rows, f32, index))
    if ws is None:
        ws = _own_ws(decode_attn_quant_ws_bytes(p, tokens, max_len, acc_out is not None), index)
    _check(lib().lrsa_decode_attn_quant(ctypes.byref(p), *args, _ws_at(ws, index), ws.nbytes, _stream_of(index)))
    return O, lse


def lrsa_cache_evict_quant(p: LrsaParams, cache: QuantCache, pos: Optional[torch.Tensor], acc: torch.Tensor, lens: torch.Tensor, max_len: int,
                           budget: int, recent: int, out: QuantCache, pos_o: Optional[torch.Tensor], acc_o: torch.Tensor, lens_o: torch.Tensor,
                           ws: Optional[torch.Tensor] = None) -> None:
    """lrsa_cache_evict from one cache in 8 bits to another of the same format and block; lens -> lens_o, [B] int32 on the device."""
    index, dev, i32, f32 = _here(acc), acc.device, torch.int32, torch.float32
    (B, _, Hkv, cap, d), _, _ = _read(p)
    kv, lst = (B, Hkv, cap, d), (B, Hkv, cap)
    args = (cache._as("cache", kv, dev), _flat("pos", pos, lst, i32, index), _flat("acc", acc, lst, f32, index), _flat("lens", lens, (B,), i32, index), max_len,
            budget, recent, out._as("out", kv, dev), _flat("pos_o", pos_o, lst, i32, index), _flat("acc_o", acc_o, lst, f32, index),
            _flat("lens_o", lens_o, (B,), i32, index))
    if ws is None:
        ws = _own_ws(cache_evict_ws_bytes(p, max_len, budget), index)
    _check(lib().lrsa_cache_evict_quant(ctypes.byref(p), *args, _ws_at(ws, index), ws.nbytes, _stream_of(index)))


def lrsa_attn_fwd(p: LrsaParams, Q, K, V, idx, O: Optional[torch.Tensor] = None,
                  lse: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """Sparse attention forward: returns (O like Q, lse [B, Hq, n] fp32)."""
    if O is None:
        O = torch.empty_strided(Q.shape, Q.stride(), dtype=Q.dtype, device=Q.device)
    if lse is None:
        lse = torch.empty((p.batch, p.heads_q, p.seq), dtype=torch.float32, device=Q.device)
    _expect_q(p, Q.device, Q=Q, O=O)
    _expect_kv(p, Q.device, K=K, V=V)
    _expect("lse", lse, (p.batch, p.heads_q, p.seq), None, torch.float32, Q.device)
    if idx is not None:
        _expect("idx", idx, (p.batch, p.heads_kv, num_scored_chunks(p), p.topk), None, torch.int32, Q.device)
    ws, nb = _workspace(p, WS_ATTN_FWD, Q.device, ws)
    _check(lib().lrsa_attn_fwd(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(idx), _ptr(O), _ptr(lse),
                               _ptr(ws), nb, _stream()))
    return O, lse


def lrsa_attn_bwd(p: LrsaParams, Q, K, V, O, dO, lse, idx, dQ=None, dK=None, dV=None,
                  ws: Optional[torch.Tensor] = None):
    """Sparse attention backward: returns (dQ like Q, dK like K, dV like V)."""
    dQ = torch.empty_strided(Q.shape, Q.stride(), dtype=Q.dtype, device=Q.device) if dQ is None else dQ
    dK = torch.empty_strided(K.shape, K.stride(), dtype=K.dtype, device=K.device) if dK is None else dK
    dV = torch.empty_strided(K.shape, K.stride(), dtype=K.dtype, device=K.device) if dV is None else dV
    _expect_q(p, Q.device, Q=Q, O=O, dO=dO, dQ=dQ)
    _expect_kv(p, Q.device, K=K, V=V, dK=dK, dV=dV)
    _expect("lse", lse, (p.batch, p.heads_q, p.seq), None, torch.float32, Q.device)
    if idx is not None:
        _expect("idx", idx, (p.batch, p.heads_kv, num_scored_chunks(p), p.topk), None, torch.int32, Q.device)
    ws, nb = _workspace(p, WS_ATTN_BWD, Q.device, ws)
    _check(lib().lrsa_attn_bwd(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(dO), _ptr(lse), _ptr(idx),
                               _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(ws), nb, _stream()))
    return dQ, dK, dV


def fill_workspace_bytes(p: LrsaParams, row_begin: int, row_end: int, which: int) -> int:
    return int(lib().lrsa_fill_workspace_bytes(ctypes.byref(p), int(row_begin), int(row_end), which))


def attn_bwd_parts(p: LrsaParams, row_begin: int, row_end: int) -> Tuple[int, int]:
    """Parts that a backward call over these rows splits the heads of a group into: (listed keys, local window)."""
    a, b = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(lib().lrsa_attn_bwd_parts(ctypes.byref(p), int(row_begin), int(row_end), ctypes.byref(a), ctypes.byref(b)))
    return a.value, b.value


class AttnPlan(ctypes.Structure):
    """Mirror of lrsa_attn_plan_info in include/lrsa.h."""
    _fields_ = [(k, ctypes.c_int32) for k in ("fwd_waves", "dq_waves", "key_waves", "slices", "gather_parts", "window_parts")]


def attn_plan(p: LrsaParams, row_begin: int = 0, row_end: Optional[int] = None, bwd_ws_bytes: Optional[int] = None) -> AttnPlan:
    """The kernels' variants that a forward and a backward call over these rows run, with a backward workspace of that size (the one
    that the size query gives)."""
    row_end = p.seq if row_end is None else row_end
    if bwd_ws_bytes is None:
        bwd_ws_bytes = workspace_bytes(p, WS_ATTN_BWD) if (row_begin, row_end) == (0, p.seq) else fill_workspace_bytes(p, row_begin, row_end, WS_ATTN_BWD)
    plan = AttnPlan()
    _check(lib().lrsa_attn_plan(ctypes.byref(p), int(row_begin), int(row_end), int(bwd_ws_bytes), ctypes.byref(plan)))
    return plan


def _fill_ws(p, row_begin, row_end, which, device, ws):
    need = fill_workspace_bytes(p, row_begin, row_end, which)
    if ws is None:
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    return ws, ws.numel() * ws.element_size()


def lrsa_attn_fwd_fill(p: LrsaParams, row_begin: int, row_end: int, Q, K, V, idx, O=None, lse=None, ws=None):
    """One filling step of the forward: Q, O hold the rows [row_begin, row_end) only; returns (O, lse)."""
    rows = row_end - row_begin
    if O is None:
        O = torch.empty_strided(Q.shape, Q.stride(), dtype=Q.dtype, device=Q.device)
    if lse is None:
        lse = torch.empty((p.batch, p.heads_q, rows), dtype=torch.float32, device=Q.device)
    shape = (p.batch, p.heads_q, rows, p.head_dim)
    for name, t in (("Q", Q), ("O", O)):
        _expect(name, t, shape, (*p.q_stride, 1), _TORCH_DTYPE.get(p.dtype), Q.device)
    _expect_kv(p, Q.device, K=K, V=V)
    _expect("lse", lse, (p.batch, p.heads_q, rows), None, torch.float32, Q.device)
    ws, nb = _fill_ws(p, row_begin, row_end, WS_ATTN_FWD, Q.device, ws)
    _check(lib().lrsa_attn_fwd_fill(ctypes.byref(p), int(row_begin), int(row_end), _ptr(Q), _ptr(K), _ptr(V), _ptr(idx),
                                    _ptr(O), _ptr(lse), _ptr(ws), nb, _stream()))
    return O, lse


def lrsa_attn_bwd_fill(p: LrsaParams, row_begin: int, row_end: int, Q, K, V, O, dO, lse, idx, dK_acc, dV_acc,
                       dQ=None, ws=None):
    """One filling step of the backward: dQ of the rows, and their share ADDED to the fp32 sums dK_acc, dV_acc."""
    rows = row_end - row_begin
    dQ = torch.empty_strided(Q.shape, Q.stride(), dtype=Q.dtype, device=Q.device) if dQ is None else dQ
    shape = (p.batch, p.heads_q, rows, p.head_dim)
    for name, t in (("Q", Q), ("O", O), ("dO", dO), ("dQ", dQ)):
        _expect(name, t, shape, (*p.q_stride, 1), _TORCH_DTYPE.get(p.dtype), Q.device)
    _expect_kv(p, Q.device, K=K, V=V)
    for name, t in (("dK_acc", dK_acc), ("dV_acc", dV_acc)):
        _expect(name, t, (p.batch, p.heads_kv, p.seq, p.head_dim), None, torch.float32, Q.device)
    _expect("lse", lse, (p.batch, p.heads_q, rows), None, torch.float32, Q.device)
    ws, nb = _fill_ws(p, row_begin, row_end, WS_ATTN_BWD, Q.device, ws)
    _check(lib().lrsa_attn_bwd_fill(ctypes.byref(p), int(row_begin), int(row_end), _ptr(Q), _ptr(K), _ptr(V), _ptr(O),
                                    _ptr(dO), _ptr(lse), _ptr(idx), _ptr(dQ), _ptr(dK_acc), _ptr(dV_acc), _ptr(ws), nb,
                                    _stream()))
    return dQ


def lrsa_attn_bwd_finish(p: LrsaParams, dK_acc, dV_acc, dK, dV):
    """fp32 sums of the filling steps -> dK, dV."""
    _expect_kv(p, dK_acc.device, dK=dK, dV=dV)
    _check(lib().lrsa_attn_bwd_finish(ctypes.byref(p), _ptr(dK_acc), _ptr(dV_acc), _ptr(dK), _ptr(dV), _stream()))
    return dK, dV


def timing_enable(on: bool) -> None:
    """Switch per-kernel HIP-event timing on (clearing earlier records) or off."""
    _check(lib().lrsa_timing_enable(1 if on else 0))


def timing_records():
    """[(kernel name, milliseconds)] of every launch recorded since timing was switched on (waits for them)."""
    L = lib()
    out = []
    name, ms = ctypes.c_char_p(), ctypes.c_float()
    for i in range(L.lrsa_timing_count()):
        _check(L.lrsa_timing_read(i, ctypes.byref(name), ctypes.byref(ms)))
        out.append((name.value.decode(), ms.value))
    return out
