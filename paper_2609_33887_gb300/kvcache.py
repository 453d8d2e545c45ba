"""ctypes binding of libbdcache (include/bdcache.h): the paged 8-bit key/value cache of a serving loop.

Argument marshalling only, as in bdcommit.py: torch tensors become the plain pointers, sizes and strides of the C ABI,
and the library's CUDA kernels do the work. There is no fallback: without the shared library every call raises.
"""

from __future__ import annotations

import ctypes
import os
import struct
from ctypes import c_int, c_int64, c_size_t, c_void_p
from typing import NamedTuple, Optional

import torch

from .bdcommit import BD_OK, BdError, _stream_handle

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libbdcache.so")

BDKV_BF16 = 1
BDKV_F16 = 16
_DT = {torch.bfloat16: BDKV_BF16, torch.float16: BDKV_F16}
_CODES = (torch.uint8, torch.float8_e4m3fn)

# bdkv_cache, bdkv_rows, bdkv_tables_args, bdkv_attention_args as laid out in include/bdcache.h
CACHE_FIELDS = struct.Struct("PPPPqiii4xqqqqqqqq")
ROWS_FIELDS = struct.Struct("Pi4xqq")
TABLES_FIELDS = struct.Struct("iiiiqqPPPPPPPPPPP")
ATTN_FIELDS = struct.Struct("Pi4xqqPi4xqqPPqi4xPPiiiiifPNP")

_lib = None


def load_library() -> ctypes.CDLL:
    """Load libbdcache.so (built in-tree by paper_2609_33887_gb300/build.py)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"libbdcache.so not found at {LIB_PATH}: build it first "
                               "(python -c 'import __graft_entry__ as g; g.build()')")
        lib = ctypes.CDLL(LIB_PATH)
        for name, res, args in (
                ("bdkv_tables", c_int, [c_void_p, c_void_p]),
                ("bdkv_write", c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_void_p]),
                ("bdkv_attention", c_int, [c_void_p, c_void_p]),
                ("bdkv_attention_workspace", c_size_t, [c_void_p, c_void_p]),
                ("bdkv_get_device_status", c_int, [c_void_p]),
                ("bdkv_shutdown", c_int, [])):
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


class KvCache(NamedTuple):
    """The cache of one layer. k, v: E4M3 codes (float8_e4m3fn or uint8) [n_pages, page_size, n_heads, head_dim] in any
    strides with head_dim contiguous; k_scale, v_scale: uint8 [n_pages, n_heads], the E8M0 scale of each page and head
    (value = code * 2^(byte - 127))."""

    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor


class KvTables(NamedTuple):
    """What kv_tables returns: kv_lens [n_seq] int32, query_start [n_seq + 1] int32, slot_map [max_tokens] int64,
    positions [max_tokens] int32, status [n_seq] int32 (0 served, 1 too few free pages, 2 table too narrow), pool [2]
    int64 (the ring's new head and tail)."""

    kv_lens: torch.Tensor
    query_start: torch.Tensor
    slot_map: torch.Tensor
    positions: torch.Tensor
    status: torch.Tensor
    pool: torch.Tensor


def kv_cache(n_pages: int, page_size: int, n_heads: int, head_dim: int, *, device="cuda") -> KvCache:
    """An empty cache in the layout that reads fastest: a page's tokens of one head next to each other."""
    def codes():
        return torch.zeros(n_pages, n_heads, page_size, head_dim, dtype=torch.uint8, device=device).transpose(1, 2)

    def scale():
        return torch.full((n_pages, n_heads), 127, dtype=torch.uint8, device=device)

    return KvCache(codes(), codes(), scale(), scale())


def _check(rc: int, where: str) -> None:
    if rc != BD_OK:
        raise BdError(rc, where)


def _same_gpu(*tensors) -> None:
    """The library is given addresses and launches on the current device, so all of them have to be there."""
    device = tensors[0].get_device()  # -1: the host
    same = device >= 0 and device == torch._C._cuda_getDevice()
    for t in tensors:
        if t.get_device() != device:
            same = False
    if not same:
        raise ValueError("all tensors must be on the current GPU")


def _cache_fields(c: KvCache) -> bytes:
    k, v, ks, vs = c
    n_pages, page_size, n_heads, dim = k.shape
    if v.shape != k.shape or ks.shape != (n_pages, n_heads) or vs.shape != ks.shape:
        raise ValueError("k and v must be [n_pages, page_size, n_heads, head_dim], their scales [n_pages, n_heads]")
    if k.dtype not in _CODES or v.dtype not in _CODES or ks.dtype != torch.uint8 or vs.dtype != torch.uint8:
        raise ValueError("codes must be float8_e4m3fn or uint8, scales uint8 (E8M0)")
    kp, kt, kh, k1 = k.stride()
    vp, vt, vh, v1 = v.stride()
    ksp, ks1 = ks.stride()
    vsp, vs1 = vs.stride()
    if k1 != 1 or v1 != 1 or (n_heads > 1 and (ks1 != 1 or vs1 != 1)):
        raise ValueError("head_dim of the codes and heads of the scales must be contiguous")
    return CACHE_FIELDS.pack(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), n_pages, page_size, n_heads, dim,
                             kp, kt, kh, vp, vt, vh, ksp, vsp)


def _rows_fields(x: torch.Tensor, name: str) -> tuple:
    strides = x.stride()
    if len(strides) != 3 or strides[2] != 1:
        raise ValueError(f"{name} must be [tokens, heads, head_dim] with head_dim contiguous")
    dtype = _DT.get(x.dtype)
    if dtype is None:
        raise ValueError(f"{name} must be bfloat16 or float16")
    return x.data_ptr(), dtype, strides[0], strides[1]


def _out_fields(x: torch.Tensor) -> tuple:
    """_rows_fields of rows that are written."""
    data, dtype, token, head = _rows_fields(x, "out")
    tokens, heads, dim = x.shape
    if tokens <= 1:
        token = heads * head + dim  # a single token's stride says nothing
    elif heads > 1 and head > token and head < (tokens - 1) * token + dim:  # (else the library sees it)
        raise ValueError("the rows of out must not overlap")
    return data, dtype, token, head


def _vector(t: torch.Tensor, dtype, n: Optional[int], name: str) -> int:
    if t.dtype is not dtype or not t.is_contiguous() or (n is not None and t.numel() != n):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor" + ("" if n is None else f" of {n}"))
    return t.data_ptr()


def _table(t: torch.Tensor, n_seq: int) -> tuple:
    shape, strides = t.shape, t.stride()
    if t.dtype is not torch.int32 or len(shape) != 2 or shape[0] != n_seq or (shape[1] > 1 and strides[1] != 1):
        raise ValueError(f"block_table must be int32 [{n_seq}, blocks] with contiguous rows")
    if n_seq > 1 and strides[0] < shape[1]:
        raise ValueError("the rows of block_table must not overlap (an expanded one: call contiguous() first)")
    # (a single row's stride may be anything)
    return t.data_ptr(), strides[0] if n_seq > 1 else max(strides[0], shape[1]), shape[1]


def _allocate_on(stream, allocate):
    """The tensors of allocate(), for a call on `stream` (None: the current one). Memory comes from that stream's pool: of
    the current one's it could still be in use there. The current stream is noted as a reader, for when it is freed."""
    if stream is None:
        return allocate()
    reader = torch.cuda.current_stream()
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()  # (0 would be a new one)
    if stream == reader:
        return allocate()
    with torch.cuda.stream(stream):
        tensors = allocate()
    for t in tensors:
        t.record_stream(reader)
    return tensors


def kv_tables(lens: torch.Tensor, new_tokens: torch.Tensor, block_table: torch.Tensor, free_pages: torch.Tensor,
              pool: torch.Tensor, *, page_size: int, max_tokens: int, stream=None) -> KvTables:
    """Pages, slots and positions for the tokens each request adds (or, where negative, gives back).

    lens, new_tokens int32 [n_seq]; block_table int32 [n_seq, max_blocks] and free_pages int32 [ring] are updated in
    place; pool int64 [2] is the ring's (head, tail), not written. max_tokens: entries of slot_map and positions, at
    least the tokens added (entries behind them are -1). A request whose status is not 0 keeps its length; query_start
    has rows for its tokens all the same, whose attention means nothing."""
    n_seq, i32, i64 = lens.numel(), torch.int32, torch.int64
    kv_lens, query_start, slot_map, positions, status, pool_out = _allocate_on(stream, lambda: (
        lens.new_empty(n_seq), lens.new_empty(n_seq + 1), pool.new_empty(max_tokens), lens.new_empty(max_tokens),
        lens.new_empty(n_seq), pool.new_empty(2)))
    table, stride, cols = _table(block_table, n_seq)
    args = TABLES_FIELDS.pack(
        n_seq, page_size, cols, max_tokens, stride, free_pages.numel(), _vector(lens, i32, n_seq, "lens"),
        _vector(new_tokens, i32, n_seq, "new_tokens"), table, _vector(free_pages, i32, None, "free_pages"),
        _vector(pool, i64, 2, "pool"), pool_out.data_ptr(), kv_lens.data_ptr(), query_start.data_ptr(),
        slot_map.data_ptr(), positions.data_ptr(), status.data_ptr())
    _same_gpu(lens, new_tokens, block_table, free_pages, pool)
    rc = load_library().bdkv_tables(args, _stream_handle(stream))
    if rc != BD_OK:
        raise BdError(rc, "bdkv_tables")
    return KvTables(kv_lens, query_start, slot_map, positions, status, pool_out)


def kv_write(k: torch.Tensor, v: torch.Tensor, slot_map: torch.Tensor, cache: KvCache, *, stream=None) -> None:
    """Quantise keys and values [tokens, n_heads, head_dim] into the cache at slot_map int64 [tokens] (negative: not
    stored). The rows of a page must be consecutive, as kv_tables lays them out. A page keeps the largest scale that its
    tokens have needed since it was begun, also of tokens taken back."""
    n = slot_map.numel()
    if k.shape != v.shape or k.shape[2:] != cache.k.shape[3:] or k.shape[1] != cache.k.shape[2] or k.shape[0] < n:
        raise ValueError("k and v must be [tokens, n_heads, head_dim] of the cache, a row for each slot")
    kf, vf = ROWS_FIELDS.pack(*_rows_fields(k, "k")), ROWS_FIELDS.pack(*_rows_fields(v, "v"))
    fields, slots = _cache_fields(cache), _vector(slot_map, torch.int64, None, "slot_map")
    _same_gpu(k, v, slot_map, *cache)
    _check(load_library().bdkv_write(fields, kf, vf, slots, n, _stream_handle(stream)), "bdkv_write")


def _attn_fields(q, out, lse, cache, block_table, kv_lens, query_start, max_q_len, max_kv_len, scale, mask_block,
                 workspace, stream) -> bytes:
    n_seq = kv_lens.numel()
    if q.shape[2:] != cache.k.shape[3:]:
        raise ValueError("q must be [tokens, n_q_heads, head_dim] of the cache")
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    table, stride, cols = _table(block_table, n_seq)
    ws, ws_bytes = (0, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    return ATTN_FIELDS.pack(
        *_rows_fields(q, "q"), *out, 0 if lse is None else lse.data_ptr(), table, stride, cols,
        _vector(kv_lens, torch.int32, n_seq, "kv_lens"), _vector(query_start, torch.int32, n_seq + 1, "query_start"),
        n_seq, q.shape[1], max_q_len, max_kv_len, mask_block,
        q.shape[2] ** -0.5 if scale is None else scale, ws, ws_bytes, _stream_handle(stream) or 0)


def kv_attention_workspace(q, cache, block_table, kv_lens, query_start, *, max_q_len, max_kv_len, mask_block=1) -> int:
    """Bytes of workspace kv_attention needs for these arguments."""
    out = (q.data_ptr(), _DT.get(q.dtype), q.shape[1] * q.shape[2], q.shape[2])
    args = _attn_fields(q, out, None, cache, block_table, kv_lens, query_start, max_q_len, max_kv_len, None, mask_block,
                        None, 0)
    return int(load_library().bdkv_attention_workspace(_cache_fields(cache), args))


def kv_attention(q: torch.Tensor, cache: KvCache, block_table: torch.Tensor, kv_lens: torch.Tensor,
                 query_start: torch.Tensor, *, max_q_len: int, max_kv_len: int, scale: Optional[float] = None,
                 mask_block: int = 1, return_lse: bool = False, out: Optional[torch.Tensor] = None, workspace=None,
                 stream=None):
    """Attention of q [tokens, n_q_heads, head_dim] over the cached tokens of each request.

    Request s holds queries query_start[s] .. query_start[s + 1], the last of its kv_lens[s] cached tokens; q has at
    least query_start[-1] rows, and rows of the result behind those are not written.
    mask_block: 0 = no mask, 1 = causal, B = causal by blocks of B queries (a window of block slots). scale defaults to
    head_dim^-0.5. Returns out (q's shape and type), or (out, lse float32 [tokens, n_q_heads])."""
    if out is None:
        out, = _allocate_on(stream, lambda: (torch.empty_like(q, memory_format=torch.contiguous_format),))
    elif out.shape != q.shape or out.dtype != q.dtype:
        raise ValueError("out must have q's shape and type")
    lse, = _allocate_on(stream, lambda: (torch.empty(q.shape[:2], dtype=torch.float32, device=q.device),)) \
        if return_lse else (None,)
    args = _attn_fields(q, _out_fields(out), lse, cache, block_table, kv_lens, query_start, max_q_len, max_kv_len, scale,
                        mask_block, workspace, stream)
    fields = _cache_fields(cache)
    _same_gpu(q, out, block_table, kv_lens, query_start, *cache, *(() if workspace is None else (workspace,)))
    _check(load_library().bdkv_attention(fields, args), "bdkv_attention")
    return (out, lse) if return_lse else out


def kv_device_status(stream=None) -> int:
    """Synchronise `stream`, then read and clear the library's device status (BD_OK, or BD_ERR_TIMEOUT)."""
    return int(load_library().bdkv_get_device_status(_stream_handle(stream)))


def kv_shutdown() -> int:
    """Free the library-owned workspaces."""
    return int(load_library().bdkv_shutdown())
