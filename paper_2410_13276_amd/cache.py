"""Binding of include/seer_cache.h: a paged cache held in 4 bits, and eviction from a cache by
accumulated attention weight.  Re-exported by the package.

    kc, vc = seer.alloc_kv_cache_q4(pages, 64, heads_kv, 128)
    seer.kv_append_q4(k, v, kc, vc, table, positions)               # the prompt's (rotated) keys and values
    k, v = seer.kv_read(kc, vc, table, positions)                   # a cached prefix back, for the prompt's next piece
    for each new token:
        seer.kv_append_q4(k1, v1, kc, vc, table, slots, inv_freq=freqs, rope_positions=positions)
        o, lse = seer.paged_attn_q4(q1, kc, vc, table, slots, inv_freq=freqs, rope_positions=positions, want_lse=True)
        seer.kv_weights(q1, kc, table, slots, lse, weights, inv_freq=freqs, rope_positions=positions)
    lengths, kept, weights = seer.kv_evict(kc, vc, table, lengths, weights, new_table, keep=2048, first=4, last=64)

kv_read, kv_weights and kv_evict take caches of alloc_kv_cache (values) as well.  Slots and positions are the same until
something is evicted.  Tensors of a call are on one GPU, which need not be the current one; work runs on that
GPU's current stream unless `stream` is given.  Results carry no autograd graph.
"""
from __future__ import annotations

import ctypes as C
import struct

import paper_2410_13276_amd as _seer

from . import decode as _d

_P = C.c_void_p
# every symbol include/seer_cache.h declares, with its ctypes signature
SIGS = {
    "seer_kv_append_q4": ([_P] * 9, C.c_int),
    "seer_kv_read": ([_P] * 7, C.c_int),
    "seer_paged_attn_q4_workspace_bytes": ([_P, _P], C.c_size_t),
    "seer_paged_attn_q4": ([_P, _P, _P, C.c_float] + [_P] * 6 + [C.c_size_t, _P], C.c_int),
    "seer_kv_weights": ([_P, _P, _P, C.c_float] + [_P] * 6, C.c_int),
    "seer_kv_evict_workspace_bytes": ([_P, C.c_int32], C.c_size_t),
    "seer_kv_evict": ([_P, _P, _P, C.c_size_t, _P], C.c_int),
}

# the header's structures, packed in one piece
_CACHE = struct.Struct("=8iqQ" + 2 * "2Q6q")   # seer_kv_cache
_TOKENS = struct.Struct("=4i7q")               # seer_kv_tokens, seer_kv_queries
_WEIGHTS = struct.Struct("=2Q4qif")            # seer_kv_weight_buf
_EVICTION = struct.Struct("=4i3Qq4i2Q4qQ")     # seer_kv_eviction

_NO_POOL = (0,) * 8


class Q4Pool:
    """Pages of keys or values in 4 bits: codes uint8 [pages, heads_kv, page_size, head_dim / 2] (element 2 i in the low half
    of byte i) and params bf16 [pages, heads_kv, page_size, head_dim / group, 2] (step, middle): code c stands for middle +
    step (c - 7.5).  Both may be transposed views ([pages, page_size, heads_kv, ..] in memory).  Their layout is looked at once,
    when the pool is made: the tensors may not be resized or transposed in place afterwards."""
    __slots__ = ("codes", "params", "shape", "group", "_strides", "_dev")

    def __init__(self, codes, params):
        t = _d._t or _seer._torch()
        cn, pn, cs, ps = codes.shape, params.shape, codes.stride(), params.stride()
        dev = codes.get_device()
        if (len(cn) != 4 or len(pn) != 5 or cn[:3] != pn[:3] or pn[4] != 2 or pn[3] < 1 or cs[3] != 1 or ps[4] != 1
                or ps[3] != 2 and pn[3] > 1 or (ps[0] | ps[1] | ps[2]) & 1 or params.get_device() != dev
                or codes.dtype is not t.uint8 or params.dtype is not t.bfloat16):
            self._refuse(codes, params)
        dim = 2 * cn[3]
        put = super().__setattr__
        put("codes", codes)
        put("params", params)
        put("shape", (cn[0], cn[1], cn[2], dim))  # [pages, heads_kv, page_size, head_dim]
        put("group", dim // pn[3])
        put("_strides", (cs[0], cs[1], cs[2], ps[0] // 2, ps[1] // 2, ps[2] // 2))
        put("_dev", dev)

    def __setattr__(self, name, value):
        raise AttributeError("a Q4Pool's tensors are given when it is made")

    @staticmethod
    def _refuse(c, p):
        torch = _seer._torch()
        if c.device != p.device:
            raise ValueError("codes and params must be on one GPU")
        if c.dtype is not torch.uint8 or p.dtype is not torch.bfloat16:
            raise TypeError("a Q4Pool holds uint8 codes and bfloat16 params")
        if c.dim() != 4 or p.dim() != 5 or c.shape[:3] != p.shape[:3] or p.shape[4] != 2 or p.shape[3] < 1:
            raise ValueError("a Q4Pool holds codes [pages, heads_kv, page_size, head_dim / 2] and params [pages, heads_kv, "
                             "page_size, head_dim / group, 2]")
        raise ValueError("a Q4Pool holds each head's codes and params contiguously")

    @property
    def head_dim(self) -> int:
        return self.shape[3]


def alloc_kv_cache_q4(num_pages: int, page_size: int, heads_kv: int, head_dim: int, group: int = 32, device="cuda"):
    """(K, V) pools in 4 bits: 5 bits an element with group 32, 4.5 with group 64, which is coarser."""
    torch = _seer._torch()
    if group not in (32, 64) or head_dim % group:
        raise ValueError("group must be 32 or 64")
    shape = (num_pages, heads_kv, page_size)
    return tuple(Q4Pool(torch.empty(*shape, head_dim // 2, dtype=torch.uint8, device=device),
                        torch.empty(*shape, head_dim // group, 2, dtype=torch.bfloat16, device=device)) for _ in range(2))


def _refuse(dev, dtype, **named):
    """Raises for the tensor that is not on GPU dev, of dtype, with unit last stride."""
    for name, t in named.items():
        if t.get_device() != dev:
            raise ValueError(f"{name} must be on the GPU of the other tensors")
        if t.dtype is not dtype:
            raise TypeError(f"{name} must be {dtype}")
        if t.stride(-1) != 1:
            raise ValueError(f"{name} must have unit last stride")


def _pool(name, pool, dev, dtype):
    """((pages, heads_kv, page_size, head_dim), group, seer_kv_pool's fields) of a Q4Pool or (group 0) a tensor of dtype."""
    if type(pool) is Q4Pool:
        if pool._dev != dev:
            raise ValueError(f"{name} must be on the GPU of the other tensors")
        return pool.shape, pool.group, (pool.codes.data_ptr(), pool.params.data_ptr(), *pool._strides)
    st = pool.stride()
    if len(st) != 4:
        raise ValueError(f"{name} must be [pages, heads_kv, page_size, head_dim] or a Q4Pool")
    if pool.get_device() != dev or (dtype is not None and pool.dtype is not dtype) or st[3] != 1:
        _refuse(dev, pool.dtype if dtype is None else dtype, **{name: pool})
    return tuple(pool.shape), 0, (pool.data_ptr(), 0, *st[:3], 0, 0, 0)


def _cache(k_cache, v_cache, table, dev, dtype, dim, heads=None, code=0):
    """seer_kv_cache (v_cache None: keys alone), its group and shape."""
    shape, group, kf = _pool("k_cache", k_cache, dev, dtype)
    vf = _NO_POOL
    if v_cache is not None:
        vshape, vgroup, vf = _pool("v_cache", v_cache, dev, dtype)
        if vshape != shape or vgroup != group:
            raise ValueError("the caches must be alike")
    if dim is not None and shape[3] != dim or heads is not None and shape[1] != heads:
        raise ValueError("the caches must be [pages, heads_kv, page_size, head_dim], heads and head_dim those of the tokens")
    n, ts = table.shape, table.stride()
    if table.dtype is not _d._t.int32 or table.get_device() != dev:
        _d._check_int("table", table, dev)
    if len(n) != 2 or ts[1] != 1 and n[1] > 1:
        raise ValueError("table must be [rows, pages] with unit last stride")
    packed = _CACHE.pack(shape[1], shape[3], code, group, shape[2], shape[0], n[0], n[1], ts[0], table.data_ptr(), *kf, *vf)
    return packed, group, shape


def _q4_only(group, name):
    if not group:
        raise TypeError(f"{name} takes caches of alloc_kv_cache_q4")


def _dtype(t):
    code = _d._code.get(t)
    if code is None:
        raise TypeError(f"unsupported dtype {t}: bfloat16 or float32")
    return code


def _same_layout(name, t, dev, batch, tokens, pos_stride):
    """Pointer of an optional tensor that is laid out like positions."""
    if t is None:
        return None
    if _d._per_token(name, t, dev, batch, tokens) != pos_stride and batch > 1:
        raise ValueError(f"{name} must be laid out like positions")
    return t.data_ptr()


def kv_append_q4(k, v, k_cache, v_cache, table, positions, *, rows=None, inv_freq=None, rope_positions=None,
                 interleaved: bool = False, rope_scale: float = 1.0, stream=None) -> None:
    """Holds the keys and values of new tokens in 4 bits (seer_kv_append_q4): token positions[b, s] of the sequence of table
    row rows[b, s], the keys rotated at rope_positions (None: positions) when inv_freq is given.  Arguments as kv_append's, the
    caches Q4Pools."""
    if _d._t is None:
        _d._load()
    if v.shape != k.shape:
        raise ValueError("k and v must be shaped alike")
    (batch, heads, tokens, dim), ks = _d._tokens_of(k, "k")
    vs = _d._tokens_of(v, "v")[1]
    dev, dtype = k.get_device(), k.dtype
    if dev < 0 or v.get_device() != dev or v.dtype is not dtype or k.stride(-1) != 1 or v.stride(-1) != 1:
        _d._refuse_tensors(dtype, k=k, v=v)
    if stream is not None or _d._device() != dev:
        with _d._elsewhere(dev, stream):
            return kv_append_q4(k, v, k_cache, v_cache, table, positions, rows=rows, inv_freq=inv_freq,
                                rope_positions=rope_positions, interleaved=interleaved, rope_scale=rope_scale)
    cache, group, _ = _cache(k_cache, v_cache, table, dev, None, dim, heads)
    _q4_only(group, "kv_append_q4")
    pos_stride = _d._per_token("positions", positions, dev, batch, tokens)
    rp = _same_layout("rows", rows, dev, batch, tokens, pos_stride)
    tp = _same_layout("rope_positions", rope_positions, dev, batch, tokens, pos_stride)
    params = _d._rope_arg(inv_freq, interleaved, rope_scale, dev)
    code = _dtype(dtype)
    if k.numel() == 0:
        return
    status = _d._fns["seer_kv_append_q4"](cache, _TOKENS.pack(batch, tokens, code, 0, *ks, *vs, pos_stride), params,
                                          k.data_ptr(), v.data_ptr(), positions.data_ptr(), tp, rp, _d._raw_stream(dev))
    if status:
        _seer._check(status, "seer_kv_append_q4")


def kv_read(k_cache, v_cache, table, positions, *, rows=None, dtype=None, out=None, stream=None):
    """What a paged cache holds for tokens (seer_kv_read): those at positions [B, S] of table row b as [B, Hkv, S, D], or those
    at positions [T] of the table rows `rows` [T] (None: row t) as [T, Hkv, D].  Padding (a negative position or row) and tokens
    without a page read as 0.  dtype: of the results, bfloat16 (None) or float32, for Q4Pools; a cache of values gives its own.  out: (k, v) to
    write to.  Returns (k, v)."""
    if _d._t is None:
        _d._load()
    dev = positions.get_device()
    if dev < 0:
        raise ValueError("positions must be on a GPU")
    if stream is not None or _d._device() != dev:
        with _d._elsewhere(dev, stream):
            return kv_read(k_cache, v_cache, table, positions, rows=rows, dtype=dtype, out=out)
    if type(k_cache) is Q4Pool:
        dtype = (out[0].dtype if out is not None else _d._t.bfloat16) if dtype is None else dtype
    else:
        if dtype is not None and dtype is not k_cache.dtype:
            raise TypeError("a cache of values is read as its own dtype")
        dtype = k_cache.dtype
    code = _dtype(dtype)
    cache, group, (_, heads, _, dim) = _cache(k_cache, v_cache, table, dev, None if type(k_cache) is Q4Pool else dtype, None,
                                              code=code)
    n = positions.shape
    if len(n) == 2:
        batch, tokens = n
        shape = (batch, heads, tokens, dim)
    elif len(n) == 1:
        batch, tokens = n[0], 1
        shape = (batch, heads, dim)
    else:
        raise ValueError("positions must be [batch, tokens] or [tokens]")
    pos_stride = _d._per_token("positions", positions, dev, batch, tokens)
    rp = _same_layout("rows", rows, dev, batch, tokens, pos_stride)
    if out is None:
        k, v = (_d._t.empty(shape, dtype=dtype, device=positions.device) for _ in range(2))
    else:
        k, v = out
        if k.shape != shape or v.shape != shape:
            raise ValueError(f"an output must be {list(shape)}")
        _refuse(dev, dtype, **{"out k": k, "out v": v})
    if k.numel() == 0:
        return k, v
    ks, vs = _d._tokens_of(k, "k")[1], _d._tokens_of(v, "v")[1]
    status = _d._fns["seer_kv_read"](cache, _TOKENS.pack(batch, tokens, code, 0, *ks, *vs, pos_stride), k.data_ptr(),
                                     v.data_ptr(), positions.data_ptr(), rp, _d._raw_stream(dev))
    if status:
        _seer._check(status, "seer_kv_read")
    return k, v


def paged_attn_q4_workspace_bytes(q, k_cache, v_cache, table) -> int:
    """Workspace of paged_attn_q4 for these shapes (0: the call would refuse them)."""
    if _d._t is None:
        _d._load()
    (batch, heads, tokens, dim), qs = _d._tokens_of(q, "q")
    cache, group, _ = _cache(k_cache, v_cache, table, q.get_device(), None, dim)
    _q4_only(group, "paged_attn_q4")
    return _d._fns["seer_paged_attn_q4_workspace_bytes"](
        cache, _TOKENS.pack(batch, heads, tokens, _dtype(q.dtype), *qs, heads * tokens * dim, tokens * dim, dim, 0))


def paged_attn_q4(q, k_cache, v_cache, table, positions, *, inv_freq=None, rope_positions=None, interleaved: bool = False,
                  rope_scale: float = 1.0, sm_scale: float = 0.0, out=None, lse=None, want_lse: bool = False,
                  workspace=None, stream=None):
    """Attention of new tokens over a paged cache held in 4 bits (seer_paged_attn_q4).  Arguments and results as
    paged_attn's, the caches Q4Pools, positions the last slot that each token sees; inv_freq: q is rotated first, at
    rope_positions (None: positions).  The keys are opened again for every 16 rows (query heads of a KV head times tokens): with more rows than
    that the call is no faster than paged_attn over bf16.  Returns (O, LSE [B, Hq, S] ([B, Hq]) or None)."""
    if _d._t is None:
        _d._load()
    (batch, heads, tokens, dim), qs = _d._tokens_of(q, "q")
    dev, dtype = q.get_device(), q.dtype
    if dev < 0 or q.stride(-1) != 1 or out is not None:
        _d._refuse_tensors(dtype, q=q, out=out)
    if stream is not None or _d._device() != dev:
        with _d._elsewhere(dev, stream):
            return paged_attn_q4(q, k_cache, v_cache, table, positions, inv_freq=inv_freq, rope_positions=rope_positions,
                                 interleaved=interleaved, rope_scale=rope_scale, sm_scale=sm_scale, out=out, lse=lse,
                                 want_lse=want_lse, workspace=workspace)
    cache, group, _ = _cache(k_cache, v_cache, table, dev, None, dim)
    _q4_only(group, "paged_attn_q4")
    if table.shape[0] != batch:
        raise ValueError("table must have a row for each batch entry")
    if out is not None and out.shape != q.shape:
        raise ValueError("out must be shaped like q")
    pos_stride = _d._per_token("positions", positions, dev, batch, tokens)
    tp = _same_layout("rope_positions", rope_positions, dev, batch, tokens, pos_stride)
    params = _d._rope_arg(inv_freq, interleaved, rope_scale, dev)
    code = _dtype(dtype)
    if lse is not None and (lse.shape != q.shape[:-1] or lse.dtype is not _d._t.float32 or lse.get_device() != dev or
                            not lse.is_contiguous()):
        raise ValueError("lse must be contiguous float32 [batch, heads, tokens] on the GPU of the other tensors")
    if workspace is not None and (workspace.get_device() != dev or not workspace.is_contiguous()):
        raise ValueError("workspace must be contiguous and on the GPU of the other tensors")
    o = _d._t.empty_like(q) if out is None else out
    if lse is None and want_lse:
        lse = _d._t.empty(q.shape[:-1], dtype=_d._t.float32, device=q.device)
    if q.numel() == 0:
        return o, lse
    desc = _TOKENS.pack(batch, heads, tokens, code, *qs, *_d._tokens_of(o, "out")[1], pos_stride)
    if workspace is None:
        need = _d._fns["seer_paged_attn_q4_workspace_bytes"](cache, desc)
        workspace = _d._t.empty(need or 1, dtype=_d._t.uint8, device=q.device)
    status = _d._fns["seer_paged_attn_q4"](cache, desc, params, sm_scale, q.data_ptr(), positions.data_ptr(), tp, o.data_ptr(),
                                           None if lse is None else lse.data_ptr(), workspace.data_ptr(),
                                           workspace.numel() * workspace.element_size(), _d._raw_stream(dev))
    if status:
        _seer._check(status, "seer_paged_attn_q4")
    return o, lse


def _check_weights(name, t, dev, batch, heads):
    if t.dtype is not _d._t.float32:
        raise TypeError(f"{name} must be float32")
    if t.get_device() != dev:
        raise ValueError(f"{name} must be on the GPU of the other tensors")
    if t.dim() != 3 or t.shape[0] != batch or t.shape[1] != heads or (t.stride(2) != 1 and t.shape[2] > 1):
        raise ValueError(f"{name} must be [{batch}, {heads}, keys] with unit last stride")


def kv_weights(q, k_cache, table, positions, lse, weights, *, decay: float = 1.0, inv_freq=None, rope_positions=None,
               interleaved: bool = False, rope_scale: float = 1.0, sm_scale: float = 0.0, out=None, stream=None):
    """Adds to weights (float32 [B, Hkv, W]; decay: what they are multiplied by first, 0: they are not read) the attention
    weight that each cached key gets from the queries (seer_kv_weights): of the heads of its group and the tokens that
    see it.  q, table, positions, inv_freq, sm_scale: those of the attention call, lse what it returned.  k_cache: a
    Q4Pool, or values of q's dtype.  Keys from W on are not counted; weights behind the last token's slot stay.  out: a
    tensor to write to instead (of weights' shape).  Returns it."""
    if _d._t is None:
        _d._load()
    (batch, heads, tokens, dim), qs = _d._tokens_of(q, "q")
    dev, dtype = q.get_device(), q.dtype
    if dev < 0 or q.stride(-1) != 1:
        _d._refuse_tensors(dtype, q=q)
    if stream is not None or _d._device() != dev:
        with _d._elsewhere(dev, stream):
            return kv_weights(q, k_cache, table, positions, lse, weights, decay=decay, inv_freq=inv_freq,
                              rope_positions=rope_positions, interleaved=interleaved, rope_scale=rope_scale, sm_scale=sm_scale,
                              out=out)
    code = _dtype(dtype)
    cache, group, (_, heads_kv, _, _) = _cache(k_cache, None, table, dev, dtype, dim, code=code)
    if table.shape[0] != batch:
        raise ValueError("table must have a row for each batch entry")
    _check_weights("weights", weights, dev, batch, heads_kv)
    if out is None:
        out = weights
    else:
        _check_weights("out", out, dev, batch, heads_kv)
        if out.shape != weights.shape:
            raise ValueError("out must be shaped like weights")
    if lse.shape != q.shape[:-1] or lse.dtype is not _d._t.float32 or lse.get_device() != dev or not lse.is_contiguous():
        raise ValueError("lse must be contiguous float32 [batch, heads, tokens] on the GPU of the other tensors")
    pos_stride = _d._per_token("positions", positions, dev, batch, tokens)
    tp = _same_layout("rope_positions", rope_positions, dev, batch, tokens, pos_stride)
    params = _d._rope_arg(inv_freq, interleaved, rope_scale, dev)
    if q.numel() == 0 or weights.numel() == 0:
        return out
    buf = _WEIGHTS.pack(weights.data_ptr(), out.data_ptr(), *weights.stride()[:2], *out.stride()[:2], weights.shape[2], decay)
    status = _d._fns["seer_kv_weights"](cache, _TOKENS.pack(batch, heads, tokens, code, *qs, 0, 0, 0, pos_stride), params, sm_scale,
                                        q.data_ptr(), positions.data_ptr(), tp, lse.data_ptr(), buf, _d._raw_stream(dev))
    if status:
        _seer._check(status, "seer_kv_weights")
    return out


def kv_evict(k_cache, v_cache, table, lengths, weights, new_table, keep: int, *, first: int = 0, last: int = 0, out=None,
             stream=None):
    """Cuts every sequence to `keep` slots of each KV head, which go to the pages of new_table (seer_kv_evict): its `first`
    first and `last` last ones, and of the others those of the largest weight, equal ones in their order.  lengths: int32
    [B], slots in use; weights: float32 [B, Hkv, W].  The pages of new_table may not be ones that the table's rows hold.
    out: (lengths int32 [B], which may be `lengths`, kept int32 [B, Hkv, keep], weights float32 [B, Hkv, W' >= keep]) to write to, the latter with 0
    behind the kept slots' weights; None: new ones, W' what new_table has room for.  Returns them; kept says which slots
    they were (-1 where a sequence had fewer).  A table with room for many more slots than the sequences hold (16384 and more of few
    heads) costs three more launches, 12 us: table[:, :n] avoids them."""
    if _d._t is None:
        _d._load()
    dev = lengths.get_device()
    if dev < 0:
        raise ValueError("lengths must be on a GPU")
    if stream is not None or _d._device() != dev:
        with _d._elsewhere(dev, stream):
            return kv_evict(k_cache, v_cache, table, lengths, weights, new_table, keep, first=first, last=last, out=out)
    if type(k_cache) is Q4Pool:
        code, dtype = _seer.BF16, None
    else:
        code, dtype = _dtype(k_cache.dtype), k_cache.dtype
    cache, group, (_, heads, page, _) = _cache(k_cache, v_cache, table, dev, dtype, None, code=code)
    _d._check_int("lengths", lengths, dev)
    if lengths.dim() != 1 or (lengths.stride(0) != 1 and lengths.shape[0] > 1):
        raise ValueError("lengths must be [batch] with unit stride")
    batch = lengths.shape[0]
    _check_weights("weights", weights, dev, batch, heads)
    _d._check_int("new_table", new_table, dev)
    if new_table.dim() != 2 or new_table.shape[0] != batch or (new_table.stride(1) != 1 and new_table.shape[1] > 1):
        raise ValueError(f"new_table must be [{batch}, pages] with unit last stride")
    if table.shape[0] < batch:
        raise ValueError("table must have a row for each sequence")
    if not 1 <= keep <= new_table.shape[1] * page:
        raise ValueError("keep must be at least 1 and at most what new_table has room for")
    if first < 0 or last < 0 or first + last > keep:
        raise ValueError("first and last must not be negative, nor more than keep together")
    if weights.shape[2] < 1:
        raise ValueError("weights must hold a key")
    if out is None:
        t = _d._t
        out = (t.empty(batch, dtype=t.int32, device=lengths.device),
               t.empty(batch, heads, keep, dtype=t.int32, device=lengths.device),
               t.empty(batch, heads, new_table.shape[1] * page, dtype=t.float32, device=lengths.device))
    new_lengths, kept, new_weights = out
    _d._check_int("out lengths", new_lengths, dev)
    _d._check_int("out kept", kept, dev)
    if new_lengths.shape != (batch,) or not new_lengths.is_contiguous():
        raise ValueError(f"out lengths must be contiguous [{batch}]")
    if kept.shape != (batch, heads, keep) or not kept.is_contiguous():
        raise ValueError(f"out kept must be contiguous [{batch}, {heads}, {keep}]")
    _check_weights("out weights", new_weights, dev, batch, heads)
    if new_weights.shape[2] < keep:
        raise ValueError("out weights must have room for keep slots")
    if batch == 0:
        return out
    desc = _EVICTION.pack(batch, keep, first, last, lengths.data_ptr(), new_lengths.data_ptr(), new_table.data_ptr(),
                          new_table.stride(0), new_table.shape[1], weights.shape[2], new_weights.shape[2], 0,
                          weights.data_ptr(), new_weights.data_ptr(), *weights.stride()[:2], *new_weights.stride()[:2],
                          kept.data_ptr())
    need = _d._fns["seer_kv_evict_workspace_bytes"](cache, batch)
    workspace = _d._t.empty(need, dtype=_d._t.uint8, device=lengths.device) if need else None
    status = _d._fns["seer_kv_evict"](cache, desc, workspace.data_ptr() if need else None, need, _d._raw_stream(dev))
    if status:
        _seer._check(status, "seer_kv_evict")
    return out
