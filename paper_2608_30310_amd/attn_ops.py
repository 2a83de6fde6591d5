"""ctypes binding of a hybrid model's full-attention layer at a prefix hit: pages
and slots from lengths, norm and rotation of queries and keys on their way into
the pages, and attention of a batch that shares a prefix (``include/gdn_attn.h``).

Argument checks and marshalling only, as in ``layer_ops``: strided token rows,
torch's current stream of the first tensor's device.  Lengths, tables, slots and
positions stay on the device, so a step that is captured once can be replayed
while they advance.  These are serving operators: no gradient is recorded.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from .binding import (AttnShape, PagesShape, QkShape, _check, _dtype_code, _need, _ptr, _seqlens, _stream, load_library)
from .layer_ops import _flat, _offsets, _on_device, _rows, _run_with_workspace


def _ints(t, name, shape, device):
    """Checks an int32 tensor."""
    if type(t) is torch.Tensor and t.dtype is torch.int32 and t.shape == shape and t.device == device and t.is_contiguous():
        return
    _need(t, name, torch.int32, device, len(shape))
    if tuple(t.shape) != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")


def _int32(x, name):
    """A number that a field of a shape holds as it is."""
    x = int(x)
    if not -2 ** 31 <= x < 2 ** 31:
        raise ValueError(f"{name} must fit 32 bits, got {x}")
    return x


def _cache(t, name, dtype, device, heads, dim):
    """Checks a cache of pages [pages, page_size, heads, dim] with dense elements; its strides."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device != device:
        raise ValueError(f"{name} must live on {device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != 4 or t.shape[2] != heads or t.shape[3] != dim:
        raise ValueError(f"{name} must be [pages, page_size, {heads}, {dim}], got {list(t.shape)}")
    s = t.stride()
    if s[3] != 1:
        raise ValueError(f"the elements of {name} must be dense")
    return s[:3]


@_on_device
def extend_pages(block_table: torch.Tensor, lens: torch.Tensor, cu_seqlens, free_pages: torch.Tensor, page_size: int,
                 cu_seqlens_host=None, first: int = 0, taken: Optional[torch.Tensor] = None,
                 table_out: Optional[torch.Tensor] = None, lens_out: Optional[torch.Tensor] = None,
                 taken_out: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
                 positions: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Room for a batch's new tokens, on torch's current stream: block tables, slots
    and positions from the lengths, with no copy to the host.

    block_table [N, W] int32: the pages of each sequence's tokens; lens [N] int32:
    the tokens it holds; ``cu_seqlens``: the new ones; free_pages [F] int32, of
    which ``taken`` [1] int32 (None = 0) are gone already.  Sequences take pages
    in their order.  Returns ``(table_out, lens_out, taken_out, slots [T],
    positions [T])``: new token i of sequence n has position first + lens[n] + i
    and slot page * page_size + row.  Where the free list ends (taken_out > F
    then) or a table row is full, entries and slots are -1.  The outputs may be
    the inputs (``table_out=block_table`` and so on: updated in place).
    """
    lib = load_library()
    device = block_table.device
    if block_table.dim() != 2:
        raise ValueError("block_table must be [N, W]")
    N, W = block_table.shape
    _ints(block_table, "block_table", (N, W), device)
    _ints(lens, "lens", (N,), device)
    _need(free_pages, "free_pages", torch.int32, device, 1)
    cu, host = _seqlens(cu_seqlens, cu_seqlens_host, device)
    if host.numel() - 1 != N:
        raise ValueError("cu_seqlens must hold N + 1 offsets")
    T = ctypes.c_int32.from_address(host.data_ptr() + 4 * N).value
    if taken is not None:
        _ints(taken, "taken", (1,), device)
    new = lambda *s: torch.empty(s, dtype=torch.int32, device=device)
    # rows behind the last new token are left alone
    def row(t, name):
        if t is None:
            return new(max(T, 0))
        _need(t, name, torch.int32, device, 1)
        if t.numel() < T:
            raise ValueError(f"{name} must hold {T} tokens")
        return t
    slots, positions = row(slots, "slots"), row(positions, "positions")
    table_out = new(N, W) if table_out is None else table_out
    lens_out = new(N) if lens_out is None else lens_out
    taken_out = new(1) if taken_out is None else taken_out
    _ints(table_out, "table_out", (N, W), device)
    _ints(lens_out, "lens_out", (N,), device)
    _ints(taken_out, "taken_out", (1,), device)
    shp = PagesShape(N, W, _int32(page_size, "page_size"), free_pages.numel(), _int32(first, "first"))
    stream = _stream(device)
    h = host.data_ptr()
    args = (ctypes.byref(shp), h, cu.data_ptr(), block_table.data_ptr(), lens.data_ptr(), free_pages.data_ptr(), _ptr(taken),
            table_out.data_ptr(), lens_out.data_ptr(), taken_out.data_ptr(), slots.data_ptr(), positions.data_ptr())
    _run_with_workspace(lambda ws, nbytes: lib.gdn_extend_pages(*args, ws, nbytes, stream),
                        lib.gdn_extend_pages_workspace_size, shp, h, device, stream, workspace)
    return table_out, lens_out, taken_out, slots, positions


@_on_device
def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, cos_sin: torch.Tensor,
                 q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                 interleaved: bool = False, v: Optional[torch.Tensor] = None, k_cache: Optional[torch.Tensor] = None,
                 v_cache: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
                 q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
    """RMS norm of every query and key head, and the position rotation, in one pass
    on torch's current stream; with a cache the keys and values go into its pages.

    q [T, Hq, D], k and v [T, Hkv, D] (bf16 or fp32, token rows may be strided),
    positions [T] int32, cos_sin [P, R] fp32: R/2 cosines, then R/2 sines of each
    position; the first R elements of a head are rotated, pairs (i, i + R/2), or
    (2 i, 2 i + 1) if ``interleaved``.  q_weight and k_weight [D] fp32, both or
    neither (None = no norm).  k_cache and v_cache [pages, page_size, Hkv, D] of
    any strides with dense elements; slots [T] int32, -1 = not written.  Returns
    ``(q_out, k_out)``; k_out is None where a cache takes the keys and no ``k_out``
    is given.  q_out may be q, and k_out k.  A token whose position is not in the
    table is left out: none of its outputs is written.
    """
    lib = load_library()
    device, dtype = q.device, q.dtype
    if q.dim() != 3 or not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise ValueError("q must be [T, Hq, D] and k [T, Hkv, D]")
    T, H, D = q.shape
    Hk = k.shape[1]
    ldq, ldk = _rows(q, "q", dtype, device, (H, D)), _rows(k, "k", dtype, device, (Hk, D))
    if k.shape[0] != T:
        raise ValueError("q and k must hold the same tokens")
    _ints(positions, "positions", (T,), device)
    _need(cos_sin, "cos_sin", torch.float32, device, 2)
    _flat(q_weight, "q_weight", (D,), device)
    _flat(k_weight, "k_weight", (D,), device)
    if (v is None) != (v_cache is None) or (v is not None and k_cache is None):
        raise ValueError("v and v_cache go together, beside k_cache")
    ldv, ks, vs, pages, page_size = Hk * D, (0, 0, 0), (0, 0, 0), 0, 0
    if k_cache is not None:
        ks = _cache(k_cache, "k_cache", dtype, device, Hk, D)
        pages, page_size = k_cache.shape[:2]
        if slots is None:
            raise TypeError("slots must be a torch.Tensor")
        _ints(slots, "slots", (T,), device)
    if v is not None:
        ldv = _rows(v, "v", dtype, device, (Hk, D))
        if v.shape[0] != T:
            raise ValueError("v must hold the same tokens as q and k")
        vs = _cache(v_cache, "v_cache", dtype, device, Hk, D)
        if v_cache.shape[:2] != k_cache.shape[:2]:
            raise ValueError("k_cache and v_cache must hold the same pages")
    ldqo, ldko = H * D, Hk * D
    if q_out is None:
        q_out = torch.empty((T, H, D), dtype=dtype, device=device)
    else:
        ldqo = _rows(q_out, "q_out", dtype, device, (H, D))
    if k_out is None and k_cache is None:
        k_out = torch.empty((T, Hk, D), dtype=dtype, device=device)
    elif k_out is not None:
        ldko = _rows(k_out, "k_out", dtype, device, (Hk, D))
    if q_out.shape[0] != T or (k_out is not None and k_out.shape[0] != T):
        raise ValueError("q_out and k_out must hold the same tokens as q")
    shp = QkShape(T, H, Hk, D, _dtype_code(q), cos_sin.shape[1], int(bool(interleaved)), cos_sin.shape[0], float(eps), pages,
                  page_size, ldq, ldk, ldv, ldqo, ldko, *ks, *vs)
    _check(lib.gdn_qk_norm_rope(ctypes.byref(shp), q.data_ptr(), k.data_ptr(), _ptr(v), positions.data_ptr(),
                                cos_sin.data_ptr(), _ptr(q_weight), _ptr(k_weight), _ptr(slots), q_out.data_ptr(),
                                _ptr(k_out), _ptr(k_cache), _ptr(v_cache), _stream(device)))
    return q_out, k_out


@_on_device
def prefix_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, block_table: torch.Tensor,
                     lens: torch.Tensor, cu_seqlens, cu_seqlens_host=None, prefix_pages: Optional[torch.Tensor] = None,
                     prefix_len: int = 0, max_len: Optional[int] = None, scale: Optional[float] = None,
                     out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of a batch whose sequences share a prefix, on torch's current
    stream: prompts, suffixes and single tokens.

    q [T, Hq, D] (bf16 or fp32, token rows may be strided), packed by
    ``cu_seqlens``; k_cache and v_cache [pages, page_size, Hkv, D] of any strides
    with dense elements (head h reads h / (Hq / Hkv)).  The first ``prefix_len``
    tokens of all sequences lie in the pages of prefix_pages [ceil(prefix_len /
    page_size)] int32, what sequence n has behind them in those of block_table
    [N, W] int32; lens [N] int32 counts the latter, the queries' own tokens
    included, which are its last: query i of q_n sees the prefix and the own
    tokens up to lens[n] - q_n + i.  A query that sees nothing gets zeros,
    one all of whose scores are -inf NaN.
    ``max_len``: no sequence holds more own tokens (default: what its table row
    has room for), a length above it counts as it.  The work is cut by it, so it
    should be given where tables are much wider than the sequences are long (64
    tokens behind 4000: 26 us, 119 without it from a table of 131072 tokens).
    ``scale`` defaults to D^-1/2.  Returns out [T, Hq, D]; its rows behind the last
    sequence are left alone.
    """
    lib = load_library()
    device, dtype = q.device, q.dtype
    if q.dim() != 3 or not isinstance(k_cache, torch.Tensor) or k_cache.dim() != 4:
        raise ValueError("q must be [T, Hq, D] and k_cache [pages, page_size, Hkv, D]")
    T, H, D = q.shape
    pages, page_size, Hk = k_cache.shape[:3]
    ldq = _rows(q, "q", dtype, device, (H, D))
    ks, vs = (_cache(t, name, dtype, device, Hk, D) for t, name in ((k_cache, "k_cache"), (v_cache, "v_cache")))
    if v_cache.shape[:2] != k_cache.shape[:2]:
        raise ValueError("k_cache and v_cache must hold the same pages")
    cu, host = _offsets(cu_seqlens, cu_seqlens_host, device, T)
    n = host.numel() - 1
    _need(block_table, "block_table", torch.int32, device, 2)
    if block_table.shape[0] != n:
        raise ValueError("block_table must be [N, W]")
    _ints(lens, "lens", (n,), device)
    if prefix_len:
        if prefix_pages is None:
            raise TypeError("prefix_pages must be a torch.Tensor")
        _need(prefix_pages, "prefix_pages", torch.int32, device, 1)
        if prefix_pages.numel() * page_size < prefix_len:
            raise ValueError("prefix_pages must hold ceil(prefix_len / page_size) pages")
    if out is None:
        out, ldo = torch.empty((T, H, D), dtype=dtype, device=device), H * D
    else:
        ldo = _rows(out, "out", dtype, device, (H, D))
        if out.shape[0] != T:
            raise ValueError("out must hold the same tokens as q")
    if max_len is not None and max_len < 1:
        raise ValueError("max_len must be at least 1")
    shp = AttnShape(n, H, Hk, D, _dtype_code(q), pages, page_size, block_table.shape[1], _int32(prefix_len, "prefix_len"),
                    0 if max_len is None else _int32(max_len, "max_len"), float(D ** -0.5 if scale is None else scale), ldq, ldo, *ks, *vs)
    stream = _stream(device)
    h = host.data_ptr()
    args = (ctypes.byref(shp), h, cu.data_ptr(), q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
            block_table.data_ptr(), lens.data_ptr(), _ptr(prefix_pages) if prefix_len else None, out.data_ptr())
    _run_with_workspace(lambda ws, nbytes: lib.gdn_prefix_attention(*args, ws, nbytes, stream),
                        lib.gdn_prefix_attention_workspace_size, shp, h, device, stream, workspace)
    return out
