"""Binding of include/seer_decode.h: rotary positions, the append to a paged key-value
cache, and attention of new tokens over it.  Re-exported by the package.

    freqs, scale = seer.rope_freqs(128, theta=500000.0)
    q, k = seer.rope(q, k, freqs)                                  # prompt: after the gate, before the attention
    kc, vc = seer.alloc_kv_cache(pages, 64, heads_kv, 128)
    seer.kv_append(k, v, kc, vc, table, positions)                 # the prompt's (rotated) keys and values
    for each new token:
        seer.kv_append(k1, v1, kc, vc, table, positions, inv_freq=freqs)
        o, _ = seer.paged_attn(q1, kc, vc, table, positions, inv_freq=freqs)

Tensors of a call are on one GPU, which need not be the current one; work runs on
that GPU's current stream unless `stream` is given.
"""
from __future__ import annotations

import ctypes as C
import math
import struct
from typing import Optional

import paper_2410_13276_amd as _seer

_P = C.c_void_p
# every symbol include/seer_decode.h declares, with its ctypes signature
SIGS = {
    "seer_rope": ([_P, _P, _P, _P, _P, _P, _P, C.c_int32, C.c_int32, _P], C.c_int),
    "seer_kv_append": ([_P] * 10, C.c_int),
    "seer_paged_attn_workspace_bytes": ([_P], C.c_size_t),
    "seer_paged_attn": ([_P, _P, C.c_float] + [_P] * 8 + [C.c_size_t, _P], C.c_int),
}

# the header's structures, packed in one piece (filling ctypes fields one by one takes 15 us)
_ROPE = struct.Struct("=Qiif4x")       # seer_rope_params
_ROPE_DESC = struct.Struct("=6i13q")   # seer_rope_desc
_CACHE_DESC = struct.Struct("=10i14q")  # seer_append_desc, seer_paged_desc


def _check_tensors(named, dtype):
    """Same device (a GPU) and type, unit last stride; returns the device."""
    device = named[0][1].device
    for name, t in named:
        if not t.is_cuda or t.device != device:
            raise ValueError(f"{name} must be on the GPU of the other tensors")
        if t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype} like the other tensors")
        if t.shape[-1] > 1 and t.stride(-1) != 1:
            raise ValueError(f"{name} must have unit last stride")
    return device


def _check_ints(name, t, device, dims):
    torch = _seer._torch()
    if t.dtype != torch.int32:
        raise TypeError(f"{name} must be int32")
    if t.device != device:
        raise ValueError(f"{name} must be on the GPU of the other tensors")
    if t.dim() not in dims or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name} must have {' or '.join(map(str, dims))} dimensions and unit last stride")


def _rope_arg(inv_freq, interleaved, scale, device):
    """seer_rope_params, or None without frequencies."""
    if inv_freq is None:
        return None
    torch = _seer._torch()
    if inv_freq.dtype != torch.float64 or inv_freq.dim() != 1 or not inv_freq.is_contiguous():
        raise TypeError("inv_freq must be a contiguous float64 vector (rope_freqs)")
    if inv_freq.device != device:
        raise ValueError("inv_freq must be on the GPU of the other tensors")
    return _ROPE.pack(inv_freq.data_ptr(), 2 * inv_freq.shape[0], int(bool(interleaved)), float(scale))


class _On:
    """Makes a call's device and stream current (nothing to do where they are), so that memory which the call
    allocates belongs to the stream that works on it."""

    def __init__(self, device, stream):
        torch = _seer._torch()
        self.guard = None
        if stream is not None:
            if stream.device != device:
                raise ValueError("the stream belongs to another device than the tensors")
            self.guard = torch.cuda.stream(stream)
        elif torch.cuda.current_device() != device.index:
            self.guard = torch.cuda.device(device)

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return _seer._torch().cuda.current_stream().cuda_stream

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def rope_freqs(rot_dim: int, theta: float = 10000.0, *, scaling: str = "none", factor: float = 1.0,
               original_len: int = 0, low: float = 1.0, high: Optional[float] = None, device="cuda"):
    """Angles per position of the rot_dim / 2 planes (float64, on `device`) and the factor on the rotated values,
    for the calls' inv_freq and rope_scale:

      none     f_p = theta^(-2p / rot_dim)
      linear   f_p / factor (position interpolation)
      ntk      base theta factor^(rot_dim / (rot_dim - 2)), which divides the slowest plane's angle by factor
      bands    planes that make more than `high` turns (4) in original_len positions as they are, those of fewer
               than `low` (1) divided by factor, the ones between in proportion
      yarn     the same with `high` 32, and the rotated values times 0.1 ln(factor) + 1 (arXiv 2309.00071)

    Any other frequencies can be passed to the calls directly."""
    torch = _seer._torch()
    if rot_dim <= 0 or rot_dim % 16:
        raise ValueError("rot_dim must be a positive multiple of 16")
    if not theta > 0 or not factor >= 1 or math.isinf(theta) or math.isinf(factor):
        raise ValueError("theta must be positive and factor at least 1, both finite")
    if scaling == "ntk":
        theta = theta * factor ** (rot_dim / (rot_dim - 2))
    f = [theta ** (-2.0 * p / rot_dim) for p in range(rot_dim // 2)]
    scale = 1.0
    if scaling == "linear":
        f = [x / factor for x in f]
    elif scaling in ("bands", "yarn"):
        if original_len <= 0:
            raise ValueError(f"scaling {scaling!r} needs original_len")
        high = (4.0 if scaling == "bands" else 32.0) if high is None else high
        if not high > low:
            raise ValueError("high must be above low")
        keep = [min(1.0, max(0.0, (original_len * x / (2 * math.pi) - low) / (high - low))) for x in f]
        f = [x * (g + (1.0 - g) / factor) for x, g in zip(f, keep)]
        if scaling == "yarn":
            scale = 0.1 * math.log(factor) + 1.0
    elif scaling not in ("none", "ntk"):
        raise ValueError(f"unknown scaling {scaling!r}")
    return torch.tensor(f, dtype=torch.float64, device=device), scale


def _token_strides(t, packed):
    """(batch, head, token) strides of [B, H, S, D], or of packed [T, H, D] as one batch entry."""
    st = t.stride()
    return (0, st[1], st[0]) if packed else st[:3]


def _rope(q, k, inv_freq, positions, start, interleaved, rope_scale, out, stream, grad):
    torch = _seer._torch()
    packed = q.dim() == 3
    if q.dim() not in (3, 4):
        raise ValueError("q must be [batch, heads, seq, head_dim] or packed [tokens, heads, head_dim]")
    if inv_freq is None:
        raise ValueError("inv_freq is required")
    qo, ko = out if out is not None else (None, None)
    if k is not None:
        want = q.shape[:1] + k.shape[1:2] + q.shape[2:]
        if k.dim() != q.dim() or k.shape != want:
            raise ValueError("k must be shaped like q, but for the heads")
    for name, o, x in (("q", qo, q), ("k", ko, k)):
        if o is not None and (x is None or o.shape != x.shape):
            raise ValueError(f"the output of {name} must be shaped like it")
    if out is not None and (qo is None or (ko is None) != (k is None)):
        raise ValueError("out must hold an output for each input")
    named = [(name, x) for name, x in (("q", q), ("k", k), ("out of q", qo), ("out of k", ko)) if x is not None]
    device = _check_tensors(named, q.dtype)
    if packed:
        (seq, heads, dim), batch = q.shape, 1
    else:
        batch, heads, seq, dim = q.shape
    pos_stride = 0
    if positions is not None:
        _check_ints("positions", positions, device, (1,) if packed else (1, 2))
        if positions.shape[-1] != seq or (positions.dim() == 2 and positions.shape[0] != batch):
            raise ValueError("positions must be [batch, seq] or [seq] (one for all), [tokens] of a packed batch")
        if positions.dim() == 2:
            pos_stride = positions.stride(0)
    params = _rope_arg(inv_freq, interleaved, rope_scale, device)
    code, kv, zero = _seer._dtype_code(q), 0 if k is None else k.shape[1], (0, 0, 0)
    with _On(device, stream) as raw:
        if out is None:
            qo = torch.empty_like(q)
            ko = None if k is None else torch.empty_like(k)
        if q.numel() == 0:
            return qo, ko
        desc = _ROPE_DESC.pack(batch, heads, kv, seq, dim, code, *_token_strides(q, packed),
                               *(zero if k is None else _token_strides(k, packed)), *_token_strides(qo, packed),
                               *(zero if k is None else _token_strides(ko, packed)), pos_stride)
        st = _seer.lib().seer_rope(desc, params, q.data_ptr(), _seer._ptr(k), qo.data_ptr(), _seer._ptr(ko),
                                   _seer._ptr(positions), int(start), grad, raw)
    _seer._check(st, "seer_rope")
    return qo, ko


def rope(q, k, inv_freq, positions=None, *, start: int = 0, interleaved: bool = False, rope_scale: float = 1.0,
         out=None, stream=None):
    """Rotary positions (seer_rope) of q and k (None: q alone), [B, H, S, D] or packed [T, H, D].  positions: int32 [B,
    S], or [S] for every batch entry ([T] packed); None: start + s.  out: (q', k') to write to, which may be (q, k).
    Returns (q', k' or None)."""
    return _rope(q, k, inv_freq, positions, start, interleaved, rope_scale, out, stream, 0)


def rope_grad(dq, dk, inv_freq, positions=None, *, start: int = 0, interleaved: bool = False, rope_scale: float = 1.0,
              out=None, stream=None):
    """The gradient's way back through rope(): gradients of the rotated tensors -> of q and k."""
    return _rope(dq, dk, inv_freq, positions, start, interleaved, rope_scale, out, stream, 1)


def alloc_kv_cache(num_pages: int, page_size: int, heads_kv: int, head_dim: int, dtype=None, device="cuda"):
    """(K, V) pools [num_pages, heads_kv, page_size, head_dim], bf16 by default.  (Pools [num_pages, page_size, heads_kv,
    head_dim] work too: pass them as t.transpose(1, 2).)"""
    torch = _seer._torch()
    shape = (num_pages, heads_kv, page_size, head_dim)
    dtype = torch.bfloat16 if dtype is None else dtype
    return tuple(torch.empty(shape, dtype=dtype, device=device) for _ in range(2))


def _check_cache(kc, vc, table, device, heads, dim):
    if kc.dim() != 4 or vc.shape != kc.shape or kc.shape[3] != dim or (heads is not None and kc.shape[1] != heads):
        raise ValueError("the caches must be [pages, heads_kv, page_size, head_dim], both alike")
    _check_ints("table", table, device, (2,))


def _tokens_of(x, name):
    """(batch, heads, tokens, dim), strides of [B, H, S, D] or [B, H, D]."""
    if x.dim() == 4:
        return x.shape, x.stride()[:3]
    if x.dim() == 3:
        b, h, d = x.shape
        return (b, h, 1, d), (x.stride(0), x.stride(1), 0)
    raise ValueError(f"{name} must be [batch, heads, tokens, head_dim] or [batch, heads, head_dim]")


def _per_token(name, t, device, batch, tokens):
    """Batch stride of int32 [batch, tokens], or [batch] where there is one token."""
    _check_ints(name, t, device, (1, 2))
    if tuple(t.shape) == (batch, tokens):
        return t.stride(0)
    if t.dim() == 1 and tokens == 1 and t.shape[0] == batch:
        return t.stride(0)
    raise ValueError(f"{name} must be [{batch}, {tokens}]")


def kv_append(k, v, k_cache, v_cache, table, positions, *, rows=None, inv_freq=None, interleaved: bool = False,
              rope_scale: float = 1.0, stream=None) -> None:
    """Writes the keys and values of new tokens to the paged cache (seer_kv_append), the keys rotated at their positions
    when inv_freq is given.  k, v: [B, Hkv, S, D], or [T, Hkv, D]; positions: int32 [B, S] ([T]); rows: the table row of
    each token, shaped like positions (None: row b of [B, Hkv, S, D], row t of [T, Hkv, D]).  Tokens with a negative
    position or row are padding."""
    if v.shape != k.shape:
        raise ValueError("k and v must be shaped alike")
    (batch, heads, tokens, dim), ks = _tokens_of(k, "k")
    vs = _tokens_of(v, "v")[1]
    device = _check_tensors((("k", k), ("v", v), ("k_cache", k_cache), ("v_cache", v_cache)), k.dtype)
    _check_cache(k_cache, v_cache, table, device, heads, dim)
    pos_stride = _per_token("positions", positions, device, batch, tokens)
    if rows is not None and _per_token("rows", rows, device, batch, tokens) != pos_stride:
        raise ValueError("rows must be laid out like positions")
    params = _rope_arg(inv_freq, interleaved, rope_scale, device)
    if k.numel() == 0:
        return
    desc = _CACHE_DESC.pack(batch, tokens, heads, dim, _seer._dtype_code(k), k_cache.shape[2], k_cache.shape[0],
                            table.shape[0], table.shape[1], 0, *ks, *vs, *k_cache.stride()[:3], *v_cache.stride()[:3],
                            table.stride(0), pos_stride)
    with _On(device, stream) as raw:
        st = _seer.lib().seer_kv_append(desc, params, k.data_ptr(), v.data_ptr(), k_cache.data_ptr(),
                                        v_cache.data_ptr(), table.data_ptr(), positions.data_ptr(), _seer._ptr(rows),
                                        raw)
    _seer._check(st, "seer_kv_append")


def _paged_desc(q, o, k_cache, v_cache, table, pos_stride):
    (batch, heads, tokens, dim), qs = _tokens_of(q, "q")
    return _CACHE_DESC.pack(batch, heads, k_cache.shape[1], tokens, dim, _seer._dtype_code(q), k_cache.shape[2],
                            k_cache.shape[0], table.shape[1], 0, *qs, *_tokens_of(o, "out")[1],
                            *k_cache.stride()[:3], *v_cache.stride()[:3], table.stride(0), pos_stride)


def paged_attn_workspace_bytes(q, k_cache, v_cache, table) -> int:
    """Workspace of paged_attn for these shapes (0: the call would refuse them)."""
    return _seer.lib().seer_paged_attn_workspace_bytes(_paged_desc(q, _seer._torch().empty_like(q), k_cache, v_cache,
                                                                   table, 0))


def paged_attn(q, k_cache, v_cache, table, positions, *, inv_freq=None, interleaved: bool = False,
               rope_scale: float = 1.0, sm_scale: float = 0.0, out=None, lse=None, want_lse: bool = False,
               workspace=None, stream=None):
    """Attention of new tokens over the paged cache (seer_paged_attn).  q: [B, Hq, S, D], or [B, Hq, D] for one token of
    each sequence; positions: int32 [B, S] ([B]): a token sees the keys up to its own position, none where that is
    negative.  inv_freq: q is rotated at its position first.  A workspace given by the caller must not serve two calls
    that may run at the same time.  Returns (O, LSE [B, Hq, S] ([B, Hq]) or None)."""
    torch = _seer._torch()
    (batch, heads, tokens, dim), _ = _tokens_of(q, "q")
    if out is not None and out.shape != q.shape:
        raise ValueError("out must be shaped like q")
    named = [("q", q), ("k_cache", k_cache), ("v_cache", v_cache)] + ([] if out is None else [("out", out)])
    device = _check_tensors(named, q.dtype)
    _check_cache(k_cache, v_cache, table, device, None, dim)
    if table.shape[0] != batch:
        raise ValueError("table must have a row for each batch entry")
    pos_stride = _per_token("positions", positions, device, batch, tokens)
    params = _rope_arg(inv_freq, interleaved, rope_scale, device)
    if lse is not None and (lse.shape != q.shape[:-1] or lse.dtype != torch.float32 or lse.device != device or
                            not lse.is_contiguous()):
        raise ValueError("lse must be contiguous float32 [batch, heads, tokens] on the GPU of the other tensors")
    if workspace is not None and (workspace.device != device or not workspace.is_contiguous()):
        raise ValueError("workspace must be contiguous and on the GPU of the other tensors")
    L = _seer.lib()
    with _On(device, stream) as raw:
        o = torch.empty_like(q) if out is None else out
        if lse is None and want_lse:
            lse = torch.empty(q.shape[:-1], dtype=torch.float32, device=device)
        if q.numel() == 0:
            return o, lse
        desc = _paged_desc(q, o, k_cache, v_cache, table, pos_stride)
        if workspace is None:
            need = L.seer_paged_attn_workspace_bytes(desc)
            workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=device)
        st = L.seer_paged_attn(desc, params, float(sm_scale), q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                               table.data_ptr(), positions.data_ptr(), o.data_ptr(), _seer._ptr(lse),
                               workspace.data_ptr(), workspace.numel() * workspace.element_size(), raw)
    _seer._check(st, "seer_paged_attn")
    return o, lse
