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
that GPU's current stream unless `stream` is given.  As with the package's other calls, results
carry no autograd graph: a training program calls rope_grad in the backward pass of a function of its own.
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


# A call's checks cost the host more than its launch, so each call tests its conditions in one expression and only
# looks for the one that failed, in these functions, when there is any.

def _refuse_tensors(dtype, **named):
    """Raises for the tensor (None: not given) that is not on the GPU of the first, of its type, with unit last stride."""
    first = next(iter(named.values()))
    for name, t in named.items():
        if t is None:
            continue
        if not t.is_cuda or t.device != first.device:
            raise ValueError(f"{name} must be on the GPU of the other tensors")
        if t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype} like the other tensors")
        if t.stride(-1) != 1:
            raise ValueError(f"{name} must have unit last stride")


def _check_int(name, t, dev):
    if t.dtype is not _t.int32:
        raise TypeError(f"{name} must be int32")
    if t.get_device() != dev:
        raise ValueError(f"{name} must be on the GPU of the other tensors")


def _rope_arg(inv_freq, interleaved, scale, dev):
    """seer_rope_params, or None without frequencies."""
    if inv_freq is None:
        return None
    if inv_freq.dtype is not _t.float64 or inv_freq.stride() != _UNIT:
        raise TypeError("inv_freq must be a contiguous float64 vector (rope_freqs)")
    if inv_freq.get_device() != dev:
        raise ValueError("inv_freq must be on the GPU of the other tensors")
    return _ROPE.pack(inv_freq.data_ptr(), 2 * inv_freq.shape[0], 1 if interleaved else 0, scale)


_UNIT, _ZERO = (1,), (0, 0, 0)

# what the first call looks up for all of them
_t = None           # torch
_code = None        # torch type -> seer_dtype
_device = None      # index of the current device
_raw_stream = None  # device index -> handle of its current stream
_fn_rope = _fn_append = _fn_paged = _fn_paged_bytes = None
_fns = {}           # name -> function, of include/seer_cache.h


def _load():
    global _t, _code, _device, _raw_stream, _fn_rope, _fn_append, _fn_paged, _fn_paged_bytes
    torch, lib = _seer._torch(), _seer.lib()
    _code = {torch.bfloat16: _seer.BF16, torch.float32: _seer.F32}
    # (where this torch offers it the handle alone: the Stream object around it takes 1 to 3 us)
    _device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
        (lambda dev: torch.cuda.current_stream(dev).cuda_stream)
    _fn_rope, _fn_append = lib.seer_rope, lib.seer_kv_append
    _fn_paged, _fn_paged_bytes = lib.seer_paged_attn, lib.seer_paged_attn_workspace_bytes
    _fns.update((name, getattr(lib, name)) for name in _seer._CACHE_SIGS)
    _t = torch


def _elsewhere(dev, stream):
    """A context that makes the stream, or else the device, current: memory which the call allocates then belongs to the
    stream that works on it."""
    if stream is None:
        return _t.cuda.device(dev)
    if stream.device.index != dev:
        raise ValueError("the stream belongs to another device than the tensors")
    return _t.cuda.stream(stream)


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


def _positions_of(t, batch, seq, packed):
    """Batch stride of rope()'s positions."""
    n, st = t.shape, t.stride()
    if n[-1:] == (seq,) and (st[-1] == 1 or seq <= 1):
        if len(n) == 1:
            return 0
        if len(n) == 2 and n[0] == batch and not packed:
            return st[0]
    raise ValueError("positions must be [batch, seq] or [seq] (one for all), [tokens] of a packed batch, with unit last "
                     "stride")


def _rope(q, k, inv_freq, positions, start, interleaved, rope_scale, out, stream, grad):
    if _t is None:
        _load()
    shape = q.shape
    if len(shape) == 4:
        batch, heads, seq, dim = shape
    elif len(shape) == 3:  # packed: one batch entry
        (seq, heads, dim), batch = shape, 1
    else:
        raise ValueError("q must be [batch, heads, seq, head_dim] or packed [tokens, heads, head_dim]")
    if inv_freq is None:
        raise ValueError("inv_freq is required")
    packed, kv = len(shape) == 3, 0
    if k is not None:
        n = k.shape
        if len(n) != len(shape) or n[0] != shape[0] or n[2:] != shape[2:]:
            raise ValueError("k must be shaped like q, but for the heads")
        kv = n[1]
        if kv and not heads:
            raise ValueError("q must have heads where k has some")
    if not -0x80000000 <= start <= 0x7fffffff:
        raise ValueError("start must be a 32-bit position")
    qo, ko = (None, None) if out is None else out
    if out is not None:
        if qo is None or (ko is None) != (k is None):
            raise ValueError("out must hold an output for each input")
        if qo.shape != shape or (k is not None and ko.shape != k.shape):
            raise ValueError("an output must be shaped like its input")
    dev, dtype, qs = q.get_device(), q.dtype, q.stride()
    ks = _ZERO if k is None else k.stride()
    if (dev < 0 or qs[-1] != 1 or out is not None
            or k is not None and (k.get_device() != dev or k.dtype is not dtype or ks[-1] != 1)):
        _refuse_tensors(dtype, q=q, k=k, out_q=qo, out_k=ko)
    if stream is not None or _device() != dev:
        with _elsewhere(dev, stream):
            return _rope(q, k, inv_freq, positions, start, interleaved, rope_scale, out, None, grad)
    pos_stride, pos = 0, None
    if positions is not None:
        _check_int("positions", positions, dev)
        pos_stride = _positions_of(positions, batch, seq, packed)
        pos = positions.data_ptr()
    params = _rope_arg(inv_freq, interleaved, rope_scale, dev)
    code = _code.get(dtype)
    if code is None:
        _seer._dtype_code(q)  # raises
    if out is None:
        qo = _t.empty_like(q)
        if k is not None:
            ko = _t.empty_like(k)
    if q.numel() == 0:
        return qo, ko
    os_, kos = qo.stride(), _ZERO if k is None else ko.stride()
    if packed:
        qs, ks, os_, kos = ((0, x[1], x[0]) for x in (qs, ks, os_, kos))
    desc = _ROPE_DESC.pack(batch, heads, kv, seq, dim, code, *qs[:3], *ks[:3], *os_[:3], *kos[:3], pos_stride)
    status = _fn_rope(desc, params, q.data_ptr(), None if k is None else k.data_ptr(), qo.data_ptr(),
                      None if k is None else ko.data_ptr(), pos, start, grad, _raw_stream(dev))
    if status:
        _seer._check(status, "seer_rope")
    return qo, ko


def rope(q, k, inv_freq, positions=None, *, start: int = 0, interleaved: bool = False, rope_scale: float = 1.0,
         out=None, stream=None):
    """Rotary positions (seer_rope) of q and k (None: q alone), [B, H, S, D] or packed [T, H, D].  positions: int32 [B,
    S], or [S] for every batch entry ([T] packed); None: start + s.  out: (q', k') to write to, which may be (q, k).
    Returns (q', k' or None), which carry no autograd graph: rope_grad is the way back."""
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


def _check_cache(kc, vc, table, dev, heads, dim):
    shape = kc.shape
    if len(shape) != 4 or vc.shape != shape or shape[3] != dim or (heads is not None and shape[1] != heads):
        raise ValueError("the caches must be [pages, heads_kv, page_size, head_dim], both alike")
    _check_int("table", table, dev)
    if table.dim() != 2 or (table.stride(1) != 1 and table.shape[1] > 1):
        raise ValueError("table must be [rows, pages] with unit last stride")


def _tokens_of(x, name):
    """(batch, heads, tokens, dim) and strides of [B, H, S, D] or [B, H, D]."""
    shape, st = x.shape, x.stride()
    if len(shape) == 4:
        return shape, st[:3]
    if len(shape) == 3:
        return (shape[0], shape[1], 1, shape[2]), (st[0], st[1], 0)
    raise ValueError(f"{name} must be [batch, heads, tokens, head_dim] or [batch, heads, head_dim]")


def _per_token(name, t, dev, batch, tokens):
    """Batch stride of int32 [batch, tokens], or [batch] where there is one token."""
    _check_int(name, t, dev)
    shape, st = t.shape, t.stride()
    if len(shape) == 2 and shape[0] == batch and shape[1] == tokens and (st[1] == 1 or tokens == 1):
        return st[0]
    if len(shape) == 1 and tokens == 1 and shape[0] == batch:
        return st[0]
    raise ValueError(f"{name} must be [{batch}, {tokens}] with unit last stride")


def kv_append(k, v, k_cache, v_cache, table, positions, *, rows=None, inv_freq=None, interleaved: bool = False,
              rope_scale: float = 1.0, stream=None) -> None:
    """Writes the keys and values of new tokens to the paged cache (seer_kv_append), the keys rotated at their positions
    when inv_freq is given.  k, v: [B, Hkv, S, D], or [T, Hkv, D]; positions: int32 [B, S] ([T]); rows: the table row of
    each token, shaped like positions (None: row b of [B, Hkv, S, D], row t of [T, Hkv, D]).  Tokens with a negative
    position or row are padding."""
    if _t is None:
        _load()
    if v.shape != k.shape:
        raise ValueError("k and v must be shaped alike")
    (batch, heads, tokens, dim), ks = _tokens_of(k, "k")
    vs = _tokens_of(v, "v")[1]
    dev, dtype, kcs, vcs = k.get_device(), k.dtype, k_cache.stride(), v_cache.stride()
    if (dev < 0 or v.get_device() != dev or k_cache.get_device() != dev or v_cache.get_device() != dev
            or v.dtype is not dtype or k_cache.dtype is not dtype or v_cache.dtype is not dtype
            or k.stride(-1) != 1 or v.stride(-1) != 1 or kcs[-1] != 1 or vcs[-1] != 1):
        _refuse_tensors(dtype, k=k, v=v, k_cache=k_cache, v_cache=v_cache)
    if stream is not None or _device() != dev:
        with _elsewhere(dev, stream):
            return kv_append(k, v, k_cache, v_cache, table, positions, rows=rows, inv_freq=inv_freq,
                             interleaved=interleaved, rope_scale=rope_scale)
    _check_cache(k_cache, v_cache, table, dev, heads, dim)
    pos_stride = _per_token("positions", positions, dev, batch, tokens)
    if rows is not None and _per_token("rows", rows, dev, batch, tokens) != pos_stride and batch > 1:
        raise ValueError("rows must be laid out like positions")
    params = _rope_arg(inv_freq, interleaved, rope_scale, dev)
    code = _code.get(dtype)
    if code is None:
        _seer._dtype_code(k)  # raises
    if k.numel() == 0:
        return
    pages, _, page_size, _ = k_cache.shape
    n_rows, max_pages = table.shape
    desc = _CACHE_DESC.pack(batch, tokens, heads, dim, code, page_size, pages, n_rows, max_pages, 0, *ks, *vs,
                            *kcs[:3], *vcs[:3], table.stride(0), pos_stride)
    status = _fn_append(desc, params, k.data_ptr(), v.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                        table.data_ptr(), positions.data_ptr(), None if rows is None else rows.data_ptr(),
                        _raw_stream(dev))
    if status:
        _seer._check(status, "seer_kv_append")


def _paged_desc(shape, qs, os_, code, k_cache, v_cache, table, pos_stride):
    pages, heads_kv, page_size, _ = k_cache.shape
    batch, heads, tokens, dim = shape
    return _CACHE_DESC.pack(batch, heads, heads_kv, tokens, dim, code, page_size, pages, table.shape[1], 0, *qs, *os_,
                            *k_cache.stride()[:3], *v_cache.stride()[:3], table.stride(0), pos_stride)


def paged_attn_workspace_bytes(q, k_cache, v_cache, table) -> int:
    """Workspace of paged_attn for these shapes (0: the call would refuse them)."""
    if _t is None:
        _load()
    shape, qs = _tokens_of(q, "q")
    _, heads, tokens, dim = shape
    desc = _paged_desc(shape, qs, (heads * tokens * dim, tokens * dim, dim), _seer._dtype_code(q), k_cache, v_cache, table,
                       0)
    return _fn_paged_bytes(desc)


def paged_attn(q, k_cache, v_cache, table, positions, *, inv_freq=None, interleaved: bool = False,
               rope_scale: float = 1.0, sm_scale: float = 0.0, out=None, lse=None, want_lse: bool = False,
               workspace=None, stream=None):
    """Attention of new tokens over the paged cache (seer_paged_attn).  q: [B, Hq, S, D], or [B, Hq, D] for one token of
    each sequence; positions: int32 [B, S] ([B]): a token sees the keys up to its own position, none where that is
    negative.  inv_freq: q is rotated at its position first.  A table much wider than the sequences need costs short ones a
    second launch: table[:, :n] avoids it.  A workspace given by the caller must not serve two calls that may run at the
    same time.  Returns (O, LSE [B, Hq, S] ([B, Hq]) or None)."""
    if _t is None:
        _load()
    shape, qs = _tokens_of(q, "q")
    batch, _, tokens, dim = shape
    dev, dtype = q.get_device(), q.dtype
    if (dev < 0 or k_cache.get_device() != dev or v_cache.get_device() != dev or k_cache.dtype is not dtype
            or v_cache.dtype is not dtype or q.stride(-1) != 1 or k_cache.stride(-1) != 1 or v_cache.stride(-1) != 1
            or out is not None):
        _refuse_tensors(dtype, q=q, k_cache=k_cache, v_cache=v_cache, out=out)
    if stream is not None or _device() != dev:
        with _elsewhere(dev, stream):
            return paged_attn(q, k_cache, v_cache, table, positions, inv_freq=inv_freq, interleaved=interleaved,
                              rope_scale=rope_scale, sm_scale=sm_scale, out=out, lse=lse, want_lse=want_lse,
                              workspace=workspace)
    _check_cache(k_cache, v_cache, table, dev, None, dim)
    if table.shape[0] != batch:
        raise ValueError("table must have a row for each batch entry")
    if out is not None and out.shape != q.shape:
        raise ValueError("out must be shaped like q")
    pos_stride = _per_token("positions", positions, dev, batch, tokens)
    params = _rope_arg(inv_freq, interleaved, rope_scale, dev)
    code = _code.get(dtype)
    if code is None:
        _seer._dtype_code(q)  # raises
    if lse is not None and (lse.shape != q.shape[:-1] or lse.dtype is not _t.float32 or lse.get_device() != dev or
                            not lse.is_contiguous()):
        raise ValueError("lse must be contiguous float32 [batch, heads, tokens] on the GPU of the other tensors")
    if workspace is not None and (workspace.get_device() != dev or not workspace.is_contiguous()):
        raise ValueError("workspace must be contiguous and on the GPU of the other tensors")
    o = _t.empty_like(q) if out is None else out
    if lse is None and want_lse:
        lse = _t.empty(q.shape[:-1], dtype=_t.float32, device=q.device)
    if q.numel() == 0:
        return o, lse
    desc = _paged_desc(shape, qs, _tokens_of(o, "out")[1], code, k_cache, v_cache, table, pos_stride)
    if workspace is None:
        need = _fn_paged_bytes(desc)
        workspace = _t.empty(need or 1, dtype=_t.uint8, device=q.device)
    status = _fn_paged(desc, params, sm_scale, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), table.data_ptr(),
                       positions.data_ptr(), o.data_ptr(), None if lse is None else lse.data_ptr(),
                       workspace.data_ptr(), workspace.numel() * workspace.element_size(), _raw_stream(dev))
    if status:
        _seer._check(status, "seer_paged_attn")
    return o, lse
