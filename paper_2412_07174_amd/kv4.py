"""The 4-bit key/value cache: binding of the scap_kv4_* entry points.  Argument marshalling only.

A decode step of one layer, its arrays on the GPU (nothing is read back, so the step can be recorded into a HIP graph)::

    cache = scap.KV4Cache(pages, kv_heads, head_dim)                  # pool and reference counts
    ws = scap.KV4Workspace(cache, seqs=B, tokens=B, heads=H, max_new=1)
    scap.kv4_reserve(cache, table, old_lens, lens, workspace=ws)      # pages for the tokens to come
    scap.kv4_append(cache, k, v, starts, table, lens)                 # quantise them into the cache
    o = scap.kv4_attention(cache, q, starts, table, lens, max_new=1, workspace=ws)
"""
from __future__ import annotations

import ctypes
import math
import struct
from typing import Optional, Tuple

import torch

from .binding import _ACT, _Args, _TORCH_CODE, KV4CacheArg, ScapError, _check, _ptr, _stream, load_library

_I32 = torch.int32


# Every call runs on `stream` (a torch stream or its handle; None: the current one).  Tensors that it is given may belong to other streams:
# ordering those, and keeping such tensors alive, is the caller's (torch.Tensor.record_stream).
def kv4_block_bytes(head_dim: int, page_tokens: int) -> int:
    return int(load_library().scap_kv4_block_bytes(head_dim, page_tokens))


class KV4Cache:
    """The pool of a 4-bit cache, uint8 [layers, pages, kv_heads, block], and refs, int32 [pages] (0: free).

    Both may be given (``pool`` of that shape, ``refs``); else they are allocated, every page free.  Nothing else is kept: the
    table and the lengths of the sequences are the caller's.
    """

    def __init__(self, pages: int, kv_heads: int, head_dim: int, *, page_tokens: int = 64, layers: int = 1, device="cuda",
                 pool: Optional[torch.Tensor] = None, refs: Optional[torch.Tensor] = None):
        block = kv4_block_bytes(head_dim, page_tokens)
        if block == 0:
            raise ValueError(f"no cache of {head_dim} channels and {page_tokens} tokens a page: channels 64 or 128, pages of "
                             "16, 32, 64, 128 or 256 tokens")
        if min(pages, kv_heads, layers) < 1:
            raise ValueError(f"pages {pages}, kv_heads {kv_heads}, layers {layers}: at least 1 each")
        shape = (layers, pages, kv_heads, block)
        a = _Args()
        if pool is None:
            pool = torch.empty(shape, dtype=torch.uint8, device=device)
        a.want(pool, "pool", shape=shape, dtype=torch.uint8)
        if refs is None:
            refs = torch.zeros(pages, dtype=_I32, device=pool.device)
        a.want(refs, "refs", shape=(pages,), dtype=_I32)
        a.on_one_gpu()
        self.pool, self.refs = pool, refs
        self.pages, self.kv_heads, self.head_dim = pages, kv_heads, head_dim
        self.page_tokens, self.layers = page_tokens, layers
        self.dev = pool.get_device()
        self.arg = KV4CacheArg(_ptr(pool), _ptr(refs), pages, kv_heads, head_dim, page_tokens, layers)
        self.ref, self.at = ctypes.byref(self.arg), ctypes.addressof(self.arg)


class KV4Workspace:
    """Caller-owned scratch for one stream, for calls of up to these sizes (scap_kv4_workspace_bytes)."""

    def __init__(self, cache: KV4Cache, *, seqs: int, tokens: int = 0, heads: int = 0, max_new: int = 0, stream=None):
        lib = load_library()
        nbytes = int(lib.scap_kv4_workspace_bytes(cache.ref, seqs, tokens, heads, max_new))
        if nbytes == 0:
            raise ScapError(-2, "scap_kv4_workspace_bytes")
        self.buf = _empty((nbytes,), torch.uint8, cache, stream)
        self.nbytes, self.dev, self.ptr = nbytes, self.buf.get_device(), self.buf.data_ptr()
        _check(lib.scap_workspace_init(_ptr(self.buf), nbytes, _stream(stream)), "scap_workspace_init")


def _cache_ok(cache) -> None:
    if type(cache) is not KV4Cache and not isinstance(cache, KV4Cache):
        raise TypeError(f"cache: expected a KV4Cache, got {type(cache).__name__}")


def _where(a: _Args, cache: KV4Cache, workspace=None) -> None:
    """Every tensor of the call on the cache's GPU."""
    a.seen.append(("cache", cache.pool))
    if workspace is not None:
        if not isinstance(workspace, KV4Workspace):
            raise TypeError("workspace: expected a KV4Workspace")
        a.seen.append(("workspace", workspace.buf))
    a.on_one_gpu()


def _table(a: _Args, table, what: str = "table") -> Tuple[int, int]:
    a.want(table, what, dtype=_I32)
    if table.dim() != 2:
        raise ValueError(f"{what}: expected [sequences, pages], got shape {tuple(table.shape)}")
    return tuple(table.shape)


def _sequences(a: _Args, starts, table, lens) -> Tuple[int, int]:
    B, S = _table(a, table)
    a.want(starts, "starts", shape=(B + 1,), dtype=_I32)
    a.want(lens, "lens", shape=(B,), dtype=_I32)
    return B, S


def _heads(t, what: str, D: int, heads: Optional[int] = None):
    """Shape and strides of a [tokens, heads, D] tensor: any strides along tokens and heads (a part of a QKV row), channels side by
    side."""
    if isinstance(t, torch.Tensor) and t.dtype in _ACT:
        shape, strides = t.shape, t.stride()
        if len(shape) == 3 and shape[2] == D and strides[2] == 1 and (heads is None or shape[1] == heads):
            return shape, strides
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what}: expected a torch.Tensor, got {type(t).__name__}")
    if t.dtype not in _ACT:
        raise TypeError(f"{what}: dtype {t.dtype}, expected {_ACT}")
    if t.dim() != 3 or t.shape[2] != D or (heads is not None and t.shape[1] != heads):
        raise ValueError(f"{what}: shape {tuple(t.shape)}, expected [tokens, {heads if heads is not None else 'heads'}, {D}]")
    raise ValueError(f"{what}: the channels must lie side by side (strides {t.stride()})")


# What a decoding loop passes on every call -- plain tensors of exactly the expected type, shape and device -- is recognised with a few
# attribute reads; whatever is not goes through _Args, which accepts the rest or names the fault.
# (Tensor.__len__ is a Python function, 1.2 us: shapes are compared instead.)
def _plain_table(table, dev: int) -> bool:
    return (type(table) is torch.Tensor and table.dtype is _I32 and table.get_device() == dev and table.dim() == 2
            and table.is_contiguous())


def _plain_list(t, shape, dev: int) -> bool:
    return (type(t) is torch.Tensor and t.dtype is _I32 and t.get_device() == dev and t.shape == shape and t.is_contiguous())


def _plain_sequences(starts, table, lens, dev: int) -> bool:
    if not _plain_table(table, dev):
        return False
    B = table.size(0)
    return _plain_list(starts, (B + 1,), dev) and _plain_list(lens, (B,), dev)


# A foreign call's arguments cost 0.17 us each to convert (4.3 us of an attention call): they go over packed, 0.9 us.
APPEND, READ, ATTENTION, RESERVE, FORK, FREE, COMPACT = range(7)
_NAMES = ("append", "read", "attention", "reserve", "fork", "free", "compact")
_pack = {n: struct.Struct(f"{n}q").pack for n in (7, 10, 12, 16, 22)}
_bits, _float = struct.Struct("i"), struct.Struct("f")
_entry = None


def _call(what: int, *words) -> None:
    global _entry
    if _entry is None:
        _entry = load_library().scap_kv4_call
    n = len(words)
    rc = _entry(what | n << 8, _pack[n](*words))   # SCAP_KV4_WORDS: the entry knows how many each call takes
    if rc != 0:
        raise ScapError(rc, "scap_kv4_" + _NAMES[what])


def _empty(shape, dtype, cache, stream) -> torch.Tensor:
    """Memory for a call's result, of the pool of the stream that the call runs on: what is freed there is not handed out to another
    stream while the call may still write it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=cache.pool.device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(getattr(stream, "cuda_stream", stream)), device=cache.pool.device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=cache.pool.device)


def _at(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


def _plain_workspace(workspace, dev: int) -> bool:
    return type(workspace) is KV4Workspace and workspace.dev == dev


def _layer(cache: KV4Cache, layer: int) -> int:
    if not 0 <= layer < cache.layers:
        raise ValueError(f"layer {layer} of a cache of {cache.layers}")
    return layer


def kv4_append(cache: KV4Cache, k: torch.Tensor, v: torch.Tensor, starts, table, lens, *, layer: int = 0, stream=None) -> None:
    """Quantises the new tokens' keys and values [T, kv_heads, D] into their pages: sequence b's are rows
    starts[b] .. starts[b + 1] - 1, at positions lens[b] - (starts[b + 1] - starts[b]) .. lens[b] - 1."""
    _cache_ok(cache)
    D = cache.head_dim
    shape, ks = _heads(k, "k", D, cache.kv_heads)
    v_shape, vs = _heads(v, "v", D, cache.kv_heads)
    if k.dtype is not v.dtype or shape != v_shape:
        raise ValueError(f"k and v: {k.dtype} {tuple(k.shape)} and {v.dtype} {tuple(v.shape)}")
    if not (_plain_sequences(starts, table, lens, cache.dev) and k.get_device() == v.get_device() == cache.dev):
        a = _Args()
        _sequences(a, starts, table, lens)
        a.seen += [("k", k), ("v", v)]
        _where(a, cache)
    B, S = table.shape
    _call(APPEND, cache.at, _layer(cache, layer), k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1], _TORCH_CODE[k.dtype], shape[0],
          starts.data_ptr(), table.data_ptr(), S, lens.data_ptr(), B, _stream(stream))


def kv4_read(cache: KV4Cache, starts, table, lens, *, tokens: int, dtype=torch.bfloat16, out=None, layer: int = 0,
             stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The keys and values [tokens, kv_heads, D] that the cache holds of the tokens that kv4_append would write."""
    _cache_ok(cache)
    if dtype not in _ACT:
        raise TypeError(f"dtype {dtype}, expected {_ACT}")
    shape = (int(tokens), cache.kv_heads, cache.head_dim)
    if shape[0] < 0:
        raise ValueError(f"tokens: {tokens}")
    if out is not None or not _plain_sequences(starts, table, lens, cache.dev):
        a = _Args()
        _sequences(a, starts, table, lens)
        if out is not None:
            for t, what in zip(out, ("k_out", "v_out")):
                a.want(t, what, shape=shape, dtype=dtype)
        _where(a, cache)
    B, S = table.shape
    k, v = out if out is not None else (_empty(shape, dtype, cache, stream) for _ in range(2))
    _call(READ, cache.at, _layer(cache, layer), k.data_ptr(), v.data_ptr(), _TORCH_CODE[dtype], shape[0], starts.data_ptr(),
          table.data_ptr(), S, lens.data_ptr(), B, _stream(stream))
    return k, v


def kv4_attention(cache: KV4Cache, q: torch.Tensor, starts, table, lens, *, scale: Optional[float] = None, causal: bool = True,
                  window: int = 0, max_new: int = 0, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                  layer: int = 0, workspace: KV4Workspace, stream=None) -> torch.Tensor:
    """out[t, h] = softmax over the cache's tokens of (scale q . k), times their values.  q is [T, heads, D].

    scale: 1 / sqrt(D) by default.  A token at position p sees j <= p (all of its sequence where not causal), and j > p - window
    where window > 0; one that sees nothing gets 0.  max_new: the most new tokens of a sequence, if known (a hint).
    lse: fp32 [T, heads], receives the log of the softmax's denominator.
    """
    _cache_ok(cache)
    D = cache.head_dim
    (T, H, _), strides = _heads(q, "q", D)
    if H == 0 or H % cache.kv_heads:
        raise ValueError(f"q: {H} heads over {cache.kv_heads} kv heads")
    if not (_plain_sequences(starts, table, lens, cache.dev) and q.get_device() == cache.dev and out is None and lse is None
            and _plain_workspace(workspace, cache.dev)):
        a = _Args()
        _sequences(a, starts, table, lens)
        a.want(out, "out", shape=(T, H, D), dtype=q.dtype, optional=True)
        a.want(lse, "lse", shape=(T, H), dtype=torch.float32, optional=True)
        a.seen.append(("q", q))
        if workspace is None:
            raise TypeError("workspace: expected a KV4Workspace")
        _where(a, cache, workspace)
    if out is None:
        out = _empty((T, H, D), q.dtype, cache, stream)
    B, S = table.shape
    scale = 1.0 / math.sqrt(D) if scale is None else float(scale)
    _call(ATTENTION, cache.at, _layer(cache, layer), q.data_ptr(), strides[0], strides[1], _TORCH_CODE[q.dtype], H, T,
          starts.data_ptr(), table.data_ptr(), S, lens.data_ptr(), B, int(max_new), _bits.unpack(_float.pack(scale))[0],
          1 if causal else 0, int(window), out.data_ptr(), _at(lse), workspace.ptr, workspace.nbytes, _stream(stream))
    return out


def _info(a: _Args, info, cache: KV4Cache, stream) -> torch.Tensor:
    a.want(info, "info", shape=(4,), dtype=_I32, optional=True)
    return _empty((4,), _I32, cache, stream) if info is None else info


def kv4_reserve(cache: KV4Cache, table, old_lens, new_lens, *, info: Optional[torch.Tensor] = None, workspace: KV4Workspace,
                stream=None) -> torch.Tensor:
    """Pages for rows that grow from old_lens to new_lens tokens; a shared, partly filled last page becomes a copy of the row's own.
    All or nothing.  Returns info, int32 [4] on the GPU: pages missing (0: done; -1: a length beyond the table), pages taken, copies
    among them, pages left."""
    _cache_ok(cache)
    dev = cache.dev
    rows = table.shape[:1] if _plain_table(table, dev) else None
    if not (rows is not None and _plain_list(old_lens, rows, dev) and _plain_list(new_lens, rows, dev)
            and _plain_list(info, (4,), dev) and _plain_workspace(workspace, dev)):
        a = _Args()
        B, S = _table(a, table)
        a.want(old_lens, "old_lens", shape=(B,), dtype=_I32)
        a.want(new_lens, "new_lens", shape=(B,), dtype=_I32)
        info = _info(a, info, cache, stream)
        if workspace is None:
            raise TypeError("workspace: expected a KV4Workspace")
        _where(a, cache, workspace)
    B, S = table.shape
    _call(RESERVE, cache.at, table.data_ptr(), S, B, old_lens.data_ptr(), new_lens.data_ptr(), info.data_ptr(), workspace.ptr,
          workspace.nbytes, _stream(stream))
    return info


def kv4_fork(cache: KV4Cache, table, lens, parents, table_out, lens_out, *, stream=None) -> None:
    """Row j of table_out shares the pages of row parents[j] of table (none where that is no row); lens_out[j] is its length.  Release
    what table_out's rows held first (kv4_free).  table_out and lens_out are memory of their own: nothing that is read."""
    _cache_ok(cache)
    dev = cache.dev
    if not (_plain_table(table, dev) and _plain_table(table_out, dev) and _plain_list(lens, table.shape[:1], dev)
            and _plain_list(parents, table_out.shape[:1], dev) and _plain_list(lens_out, table_out.shape[:1], dev)):
        a = _Args()
        B, S = _table(a, table)
        B_out, S_out = _table(a, table_out, "table_out")
        a.want(lens, "lens", shape=(B,), dtype=_I32)
        a.want(parents, "parents", shape=(B_out,), dtype=_I32)
        a.want(lens_out, "lens_out", shape=(B_out,), dtype=_I32)
        _where(a, cache)
    B, S = table.shape
    B_out, S_out = table_out.shape
    if S_out != S:
        raise ValueError(f"table_out: rows of {S_out} pages, table has {S}")
    try:
        _call(FORK, cache.at, table.data_ptr(), lens.data_ptr(), B, parents.data_ptr(), B_out, table_out.data_ptr(), lens_out.data_ptr(), S,
              _stream(stream))
    except ScapError as e:
        if e.status != -5:
            raise
        raise ValueError("table_out and lens_out: overlap table, lens or parents, or each other") from None


def kv4_free(cache: KV4Cache, table, keep_from=None, keep_to=None, *, stream=None) -> None:
    """Releases the pages of table's rows that hold no token of [keep_from, keep_to): whole rows by default.  keep_to alone keeps
    the tokens before it, keep_from alone those from there on."""
    _cache_ok(cache)
    if not (keep_from is None and keep_to is None and _plain_table(table, cache.dev)):
        a = _Args()
        B, S = _table(a, table)
        a.want(keep_from, "keep_from", shape=(B,), dtype=_I32, optional=True)
        a.want(keep_to, "keep_to", shape=(B,), dtype=_I32, optional=True)
        _where(a, cache)
    B, S = table.shape
    _call(FREE, cache.at, table.data_ptr(), S, B, _at(keep_from), _at(keep_to), _stream(stream))


def kv4_compact(cache: KV4Cache, table, *, table_out=None, refs_out=None, info: Optional[torch.Tensor] = None,
                workspace: KV4Workspace, stream=None) -> torch.Tensor:
    """Moves the live pages to the front of the pool; table holds every row that names one.  Works in place unless table_out and
    refs_out are given.  Returns info, int32 [4] on the GPU: live pages, pages moved, 0, 0."""
    _cache_ok(cache)
    dev = cache.dev
    if (table_out is None) != (refs_out is None):
        raise ValueError("table_out and refs_out: both or neither")
    if not (_plain_table(table, dev) and (table_out is None or _plain_table(table_out, dev) and table_out.shape == table.shape
                                          and _plain_list(refs_out, (cache.pages,), dev))
            and _plain_list(info, (4,), dev) and _plain_workspace(workspace, dev)):
        a = _Args()
        B, S = _table(a, table)
        a.want(table_out, "table_out", shape=(B, S), dtype=_I32, optional=True)
        a.want(refs_out, "refs_out", shape=(cache.pages,), dtype=_I32, optional=True)
        info = _info(a, info, cache, stream)
        if workspace is None:
            raise TypeError("workspace: expected a KV4Workspace")
        _where(a, cache, workspace)
    B, S = table.shape
    _call(COMPACT, cache.at, table.data_ptr(), S, B, (table if table_out is None else table_out).data_ptr(),
          (cache.refs if refs_out is None else refs_out).data_ptr(), info.data_ptr(), workspace.ptr, workspace.nbytes,
          _stream(stream))
    return info


def kv4_copy_pages(cache: KV4Cache, src, dst, *, to: Optional[KV4Cache] = None, stream=None) -> None:
    """Copies page src[i] of cache to page dst[i] of `to` (default: the same cache), all layers.  No dst is another pair's page."""
    _cache_ok(cache)
    to = cache if to is None else to
    _cache_ok(to)
    a = _Args()
    a.want(src, "src", dtype=_I32)
    a.want(dst, "dst", dtype=_I32)
    if src.dim() != 1 or src.shape != dst.shape:
        raise ValueError(f"src and dst: shapes {tuple(src.shape)} and {tuple(dst.shape)}")
    a.seen.append(("to", to.pool))
    _where(a, cache)
    rc = load_library().scap_kv4_copy_pages(cache.ref, to.ref, _ptr(src), _ptr(dst), src.shape[0], _stream(stream))
    _check(rc, "scap_kv4_copy_pages")
