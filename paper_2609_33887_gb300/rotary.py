"""ctypes binding of libbdrotary (include/bdrotary.h): rotary positions on the way into the caches, and the latent cache.

Argument marshalling only, as in kvcache.py, whose conventions hold here. There is no fallback: without the shared library
every call raises.
"""

from __future__ import annotations

import ctypes
import math
import os
import struct
from ctypes import c_int, c_int32, c_int64, c_size_t, c_void_p
from fractions import Fraction
from typing import NamedTuple, Optional

import torch

from .bdcommit import BD_OK, BdError, _stream_handle
from .kvcache import (_DT, ROWS_FIELDS, KvCache, _allocate_on, _cache_fields, _check, _out_fields, _rows_fields, _same_gpu,
                      _table, _vector)

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libbdrotary.so")

# bdrot_rotary, bdrot_latent, bdrot_latent_attention_args as laid out in include/bdrotary.h
ROTARY_FIELDS = struct.Struct("Piid")
LATENT_FIELDS = struct.Struct("PPiiqiiqqqq")
LATENT_ATTN_FIELDS = struct.Struct("Pi4xqqPi4xqqPPqi4xPPiiiiifPNP")

_TURN = 2 * Fraction(3141592653589793238462643383279502884197, 10 ** 39)  # 2 pi

_lib = None


def load_library() -> ctypes.CDLL:
    """Load libbdrotary.so (built in-tree by paper_2609_33887_gb300/build.py)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"libbdrotary.so not found at {LIB_PATH}: build it first "
                               "(python -c 'import __graft_entry__ as g; g.build()')")
        lib = ctypes.CDLL(LIB_PATH)
        p = c_void_p
        for name, res, args in (
                ("bdrot_rotate", c_int, [p, p, p, c_int32, c_int32, p, c_int64, c_int32, p]),
                ("bdrot_write", c_int, [p, p, p, p, p, p, c_int64, p, p, c_int32, p]),
                ("bdrot_latent_write", c_int, [p, p, p, p, p, p, c_int64, p]),
                ("bdrot_latent_attention", c_int, [p, p]),
                ("bdrot_latent_attention_workspace", c_size_t, [p, p]),
                ("bdrot_get_device_status", c_int, [p]),
                ("bdrot_shutdown", c_int, [])):
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


class KvRotary(NamedTuple):
    """A rotation by positions, as kv_rotary makes it. turns: int64 [dim / 2], the angle a position of each pair as a
    fraction of a turn, times 2^64 (modulo 2^64); scale: what cosines and sines are multiplied by; interleaved: pairs are
    elements 2p and 2p + 1, else p and p + dim / 2, of a row's first dim elements."""

    turns: torch.Tensor
    scale: float = 1.0
    interleaved: bool = False


class KvLatent(NamedTuple):
    """The latent cache of one layer. latent: bfloat16 or float16 [n_pages, page_size, latent_dim], rope: [n_pages,
    page_size, rope_dim] of the same type, each in any strides with its last dimension contiguous (multiples of 8)."""

    latent: torch.Tensor
    rope: torch.Tensor


def kv_rotary(dim: int, *, base: float = 10000.0, frequencies=None, factor: float = 1.0, original_len: Optional[int] = None,
              slow: float = 1.0, fast: float = 32.0, scale: float = 1.0, interleaved: bool = False,
              device="cuda") -> KvRotary:
    """The rotation of a row's first `dim` elements (a multiple of 16) with frequencies base^(-2p / dim), or the given
    ones (radians a position, dim / 2 of them).

    factor: contexts stretched by it. Without original_len all frequencies are divided by it. With original_len (the
    length that the model was trained on) only those that turn at most `slow` times in it; those that turn `fast` times or
    more are kept, and in between the kept share grows linearly with the number of turns: (turns - slow) / (fast - slow).
    Models that blend by the pair's index between the two bounds instead (linearly in the logarithm of the turns) have other
    frequencies there with the same numbers: pass theirs as `frequencies`, with factor 1. scale: what the rotated elements
    are multiplied by, 1 or the amplitude that goes with the stretch."""
    if dim < 16 or dim % 16:
        raise ValueError("dim must be a positive multiple of 16")
    if frequencies is None:
        f = [float(base) ** (-2.0 * p / dim) for p in range(dim // 2)]
    else:
        f = [float(x) for x in (frequencies.tolist() if isinstance(frequencies, torch.Tensor) else frequencies)]
        if len(f) != dim // 2:
            raise ValueError(f"frequencies must be {dim // 2} numbers")
    if not (factor > 0 and math.isfinite(factor) and all(map(math.isfinite, f))):
        raise ValueError("factor must be positive, frequencies finite")
    if original_len is None:
        f = [x / factor for x in f]
    else:
        if not 0 <= slow < fast:
            raise ValueError("slow must be below fast")
        kept = [min(max((original_len * abs(x) / (2 * math.pi) - slow) / (fast - slow), 0.0), 1.0) for x in f]
        f = [x * k + x / factor * (1 - k) for x, k in zip(f, kept)]
    turns = [round(Fraction(x) / _TURN * (1 << 64)) % (1 << 64) for x in f]
    turns = torch.tensor([t - (1 << 64) if t >> 63 else t for t in turns], dtype=torch.int64, device=device)
    return KvRotary(turns, float(scale), bool(interleaved))


def kv_latent_cache(n_pages: int, page_size: int, latent_dim: int, rope_dim: int, *, dtype=torch.bfloat16,
                    device="cuda") -> KvLatent:
    """An empty latent cache in the layout that reads fastest: a token's latent and key part next to each other."""
    rows = torch.zeros(n_pages, page_size, latent_dim + rope_dim, dtype=dtype, device=device)
    return KvLatent(*rows.split([latent_dim, rope_dim], 2))


def _rotary_fields(r: KvRotary) -> bytes:
    turns, scale, interleaved = r
    if turns.dtype is not torch.int64 or not turns.is_contiguous():
        raise ValueError("turns must be a contiguous torch.int64 tensor")
    return ROTARY_FIELDS.pack(turns.data_ptr(), 2 * turns.numel(), bool(interleaved), scale)


def _latent_fields(c: KvLatent) -> bytes:
    latent, rope = c
    shape, rope_shape, dtype = latent.shape, rope.shape, _DT.get(latent.dtype)
    if len(shape) != 3 or len(rope_shape) != 3 or rope_shape[:2] != shape[:2] or rope.dtype is not latent.dtype or dtype is None:
        raise ValueError("latent and rope must be bfloat16 or float16, [n_pages, page_size, latent_dim] and "
                         "[n_pages, page_size, rope_dim]")
    lp, lt, l1 = latent.stride()
    rp, rt, r1 = rope.stride()
    if l1 != 1 or r1 != 1:
        raise ValueError("the last dimension of latent and rope must be contiguous")
    n_pages, page_size, dim = shape
    return LATENT_FIELDS.pack(latent.data_ptr(), rope.data_ptr(), dtype, page_size, n_pages, dim, rope_shape[2], lp, lt, rp,
                              rt)


def _turned_fields(x, shape, out, name, stream):
    """Rows and where they go turned (allocated where out is None): their fields and the output."""
    if out is None:
        if stream is None:
            out = torch.empty_like(x, memory_format=torch.contiguous_format)
        else:
            out, = _allocate_on(stream, lambda: (torch.empty_like(x, memory_format=torch.contiguous_format),))
    elif out.shape != shape or out.dtype is not x.dtype:
        raise ValueError(f"out must have {name}'s shape and type")
    dtype, n = _DT.get(x.dtype), shape[0]
    if dtype is None:
        raise ValueError(f"{name} must be bfloat16 or float16")
    if n == 0:
        none = ROWS_FIELDS.pack(0, dtype, 0, 0)
        return none, none, out
    (token, head, one), (o_token, o_head, o_one) = x.stride(), out.stride()
    if one != 1 or o_one != 1:
        raise ValueError(f"{name} and out must be [tokens, heads, head_dim] with head_dim contiguous")
    if n == 1:  # (the strides of a single token, or head, say nothing)
        token = o_token = 0
    if shape[1] == 1:
        head = o_head = 0
    return (ROWS_FIELDS.pack(x.data_ptr(), dtype, token, head), ROWS_FIELDS.pack(out.data_ptr(), dtype, o_token, o_head),
            out)


def kv_rotate(x: torch.Tensor, positions: torch.Tensor, rotary: KvRotary, *, inverse: bool = False,
              out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """x [tokens, heads, head_dim] with the first elements of each head turned by positions int32 [tokens].

    inverse: turned back, with the same scale (the adjoint: gradients of the result to gradients of x). out may be x; to
    turn the last elements of a head, pass x[..., first:] for both. Returns out."""
    shape = x.shape
    if len(shape) != 3:
        raise ValueError("x must be [tokens, heads, head_dim] with head_dim contiguous")
    n, heads, dim = shape
    xf, of, out = _turned_fields(x, shape, out, "x", stream)
    fields, pos = _rotary_fields(rotary), _vector(positions, torch.int32, n, "positions")
    _same_gpu(x, positions, rotary[0], out)
    rc = load_library().bdrot_rotate(fields, xf, of, heads, dim, pos, n, bool(inverse), _stream_handle(stream))
    if rc != BD_OK:
        raise BdError(rc, "bdrot_rotate")
    return out


def kv_write_rotated(k: torch.Tensor, v: torch.Tensor, slot_map: torch.Tensor, cache: KvCache, positions: torch.Tensor,
                     rotary: KvRotary, *, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                     stream=None) -> Optional[torch.Tensor]:
    """kv_write of keys turned by positions int32 (a position for each slot), and queries turned in the same call.

    The cache gets the codes and scales of kv_write(kv_rotate(k), v). q: [tokens, n_q_heads, head_dim], a row for each
    slot; q_out may be q. Returns the turned queries (None without q)."""
    n, shape, (_, _, heads, dim) = slot_map.numel(), k.shape, cache.k.shape
    if len(shape) != 3 or shape != v.shape or shape[2] != dim or shape[1] != heads or shape[0] < n:
        raise ValueError("k and v must be [tokens, n_heads, head_dim] of the cache, a row for each slot")
    kf, vf = ROWS_FIELDS.pack(*_rows_fields(k, "k")), ROWS_FIELDS.pack(*_rows_fields(v, "v"))
    fields, slots = _cache_fields(cache), _vector(slot_map, torch.int64, None, "slot_map")
    pos, rf = _vector(positions, torch.int32, n, "positions"), _rotary_fields(rotary)
    if q is None:
        if q_out is not None:
            raise ValueError("q_out without q")
        qf, of, n_q = None, None, 0
        _same_gpu(k, v, slot_map, positions, rotary[0], *cache)
    else:
        q_shape = q.shape
        if len(q_shape) != 3 or q_shape[0] != n or q_shape[2] != dim:
            raise ValueError("q must be [tokens, n_q_heads, head_dim] of the cache, a row for each slot")
        qf, of, q_out = _turned_fields(q, q_shape, q_out, "q", stream)
        n_q = q_shape[1]
        _same_gpu(k, v, slot_map, positions, rotary[0], q, q_out, *cache)
    rc = load_library().bdrot_write(rf, fields, kf, vf, slots, pos, n, qf, of, n_q, _stream_handle(stream))
    if rc != BD_OK:
        raise BdError(rc, "bdrot_write")
    return q_out


def _vectors_fields(x, dim, n, dtype, name):
    shape = x.shape
    if len(shape) != 2 or shape[0] < n or shape[1] != dim or x.dtype is not dtype:
        raise ValueError(f"{name} must be [tokens, {dim}] of the cache's type, a row for each slot")
    token, one = x.stride()
    if one != 1 and shape[0]:
        raise ValueError(f"the rows of {name} must be contiguous")
    return ROWS_FIELDS.pack(x.data_ptr(), _DT[dtype], token if shape[0] > 1 else 0, 0)


def kv_latent_write(latent: torch.Tensor, rope: torch.Tensor, slot_map: torch.Tensor, cache: KvLatent, *,
                    positions: Optional[torch.Tensor] = None, rotary: Optional[KvRotary] = None, stream=None) -> None:
    """Latents [tokens, latent_dim] and key parts [tokens, rope_dim] into the cache at slot_map int64 [tokens] (negative:
    not stored; no slot twice). With rotary (of rope_dim elements), key parts are turned by positions int32 [tokens].
    Without it they are stored as they are."""
    n, dtype = slot_map.numel(), cache[0].dtype
    fields = _latent_fields(cache)
    lf = _vectors_fields(latent, cache[0].shape[2], n, dtype, "latent")
    rf = _vectors_fields(rope, cache[1].shape[2], n, dtype, "rope")
    slots = _vector(slot_map, torch.int64, None, "slot_map")
    if (positions is None) != (rotary is None):
        raise ValueError("positions and rotary go together")
    if rotary is None:
        turn = pos = None
        _same_gpu(latent, rope, slot_map, *cache)
    else:
        turn, pos = _rotary_fields(rotary), _vector(positions, torch.int32, n, "positions")
        _same_gpu(latent, rope, slot_map, positions, rotary[0], *cache)
    _check(load_library().bdrot_latent_write(turn, fields, lf, rf, slots, pos, n, _stream_handle(stream)),
           "bdrot_latent_write")


def _latent_attn_fields(q, shape, out, lse, cache, block_table, kv_lens, query_start, max_q_len, max_kv_len, scale,
                        mask_block, workspace, stream) -> bytes:
    n_seq = kv_lens.numel()
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    table, stride, cols = _table(block_table, n_seq)
    ws, ws_bytes = (0, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    return LATENT_ATTN_FIELDS.pack(
        *_rows_fields(q, "q"), *out, 0 if lse is None else lse.data_ptr(), table, stride, cols,
        _vector(kv_lens, torch.int32, n_seq, "kv_lens"), _vector(query_start, torch.int32, n_seq + 1, "query_start"),
        n_seq, shape[1], max_q_len, max_kv_len, mask_block, scale, ws, ws_bytes, _stream_handle(stream) or 0)


def _latent_q(q, cache):
    """(q's shape, latent_dim)."""
    shape, dim = q.shape, cache[0].shape[2]
    if len(shape) != 3 or shape[2] != dim + cache[1].shape[2] or q.dtype is not cache[0].dtype:
        raise ValueError("q must be [tokens, heads, latent_dim + rope_dim] of the cache's type")
    return shape, dim


def kv_latent_attention_workspace(q, cache, block_table, kv_lens, query_start, *, max_q_len, max_kv_len) -> int:
    """Bytes of workspace kv_latent_attention needs for these arguments."""
    shape, dim = _latent_q(q, cache)
    out = (q.data_ptr(), _DT.get(q.dtype), shape[1] * dim, dim)
    args = _latent_attn_fields(q, shape, out, None, cache, block_table, kv_lens, query_start, max_q_len, max_kv_len, 1.0, 0,
                               None, 0)
    return int(load_library().bdrot_latent_attention_workspace(_latent_fields(cache), args))


def _apart(q, out) -> None:
    """Refuses an output that lies on the queries, which other rows' work still reads: exact where the two have the same
    strides (those of one token or one head aside), else whether their addresses meet."""
    (n, heads, wide), dim, (token, head, _), (o_token, o_head, _) = q.shape, out.shape[2], q.stride(), out.stride()
    if not q.numel() or not out.numel():
        return

    def end(t):
        return t.data_ptr() + 2 * (1 + sum((s - 1) * x for s, x in zip(t.shape, t.stride())))

    if q.data_ptr() >= end(out) or out.data_ptr() >= end(q):
        return
    if (n == 1 or token == o_token) and (heads == 1 or head == o_head):
        gap = (out.data_ptr() - q.data_ptr()) // 2
        if heads > 1 and head > 0 and (n == 1 or token % head == 0) and wide <= gap % head <= head - dim:
            return  # each head's result behind its queries
        step, most = (token, n - 1) if n > 1 and token > 0 else (1 << 62, 0)
        for d in range(1 - heads, heads):  # a head of out less one of q, and k tokens: -dim < x + k * step < wide?
            x = gap + d * head
            if max(-((x + dim - 1) // step), -most) <= min((wide - 1 - x) // step, most):
                break
        else:
            return
    raise ValueError("out must not lie on q")


def kv_latent_attention(q: torch.Tensor, cache: KvLatent, block_table: torch.Tensor, kv_lens: torch.Tensor,
                        query_start: torch.Tensor, *, scale: float, max_q_len: int, max_kv_len: int, mask_block: int = 1,
                        return_lse: bool = False, out: Optional[torch.Tensor] = None, workspace=None, stream=None):
    """Attention of q [tokens, heads, latent_dim + rope_dim] over the cached latents of each request: every head's keys
    are the cached latents and key parts, its values the latents.

    Requests, masks, bounds, workspace and rows behind the last query are as in kv_attention. scale has no default: it is
    the one of the heads before their projection into the latent's space. Returns out [tokens, heads, latent_dim] of q's
    type, or (out, lse float32 [tokens, heads])."""
    shape, dim = _latent_q(q, cache)
    n, heads, _ = shape
    if out is None:
        if stream is None:
            out = q.new_empty((n, heads, dim))
        else:
            out, = _allocate_on(stream, lambda: (q.new_empty((n, heads, dim)),))
        out_fields = out.data_ptr(), _DT.get(q.dtype), heads * dim, dim
    else:
        if out.shape != (n, heads, dim) or out.dtype != q.dtype:
            raise ValueError("out must be [tokens, heads, latent_dim] of q's type")
        out_fields = _out_fields(out)
        _apart(q, out)
    lse, = _allocate_on(stream, lambda: (q.new_empty((n, heads), dtype=torch.float32),)) if return_lse else (None,)
    _same_gpu(q, out, block_table, kv_lens, query_start, *cache, *(() if workspace is None else (workspace,)))
    args = _latent_attn_fields(q, shape, out_fields, lse, cache, block_table, kv_lens, query_start, max_q_len,
                               max_kv_len, scale, mask_block, workspace, stream)
    rc = load_library().bdrot_latent_attention(_latent_fields(cache), args)
    if rc != BD_OK:
        raise BdError(rc, "bdrot_latent_attention")
    return (out, lse) if return_lse else out


def kv_latent_device_status(stream=None) -> int:
    """Synchronise `stream`, then read and clear the library's device status (BD_OK, or BD_ERR_TIMEOUT)."""
    return int(load_library().bdrot_get_device_status(_stream_handle(stream)))


def kv_latent_shutdown() -> int:
    """Free the library-owned workspaces."""
    return int(load_library().bdrot_shutdown())
