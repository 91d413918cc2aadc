"""A paged key/value cache: torch faces of the calls of include/tlinpaged.h.

Caches are ``[num_pages, key heads, page rows, D]`` tensors (any strides with whole 16-byte pieces, so a view of
``[num_pages, page rows, key heads, D]`` is one too), new rows ``[heads, T, D]`` (a view of ``[T, heads, D]`` is one), and
the table, lengths, starts and counts int32 tensors on the same device.  Nothing here synchronises.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding
from .binding import (BOOK_LAYOUT, CACHE_LAYOUT, PAGED_LAYOUT, ROPE_LAYOUT, TLIN_BF16, TLIN_F32, TlinBookParams,
                      TlinCacheParams, TlinPagedParams, TlinRopeParams, packed)

_CODES = {torch.float32: TLIN_F32, torch.bfloat16: TLIN_BF16}
_SCALINGS = {None: 0, "linear": 1, "base": 2, "parts": 3}


def _code(dtype):
    try:
        return _CODES[dtype]
    except KeyError:
        raise TypeError(f"unsupported dtype {dtype}: float32 or bfloat16 expected") from None


def _check(device, dtype=None, **tensors):
    """Every tensor that is there on the device, the rows of one type."""
    for name, t in tensors.items():
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError(f"{name}: libtlinattn takes device tensors only")
        if t.device != device:
            raise ValueError(f"{name} is on {t.device}, the call on {device}")
        if dtype is not None and t.dtype != dtype:
            raise TypeError(f"{name} is {t.dtype}, {dtype} expected")


def _flat(device, size, **tensors):
    """int32 vectors on the device, at least `size` long."""
    for name, t in tensors.items():
        if t.dtype != torch.int32 or t.device != device:
            raise TypeError(f"{name}: an int32 tensor on {device} expected, not {t.dtype} on {t.device}")
        if t.dim() != 1 or t.shape[0] < size or (t.shape[0] > 1 and t.stride(0) != 1):
            raise ValueError(f"{name}: {size} entries, one after another, expected")


def _rows(t, axes, name):
    st = t.stride()
    if len(st) != axes or (st[-1] != 1 and t.shape[-1] != 1):
        raise ValueError(f"{name}: {axes} axes expected, the last one contiguous")
    return st[:-1]


def _like(t, dtype=None):
    """An uninitialised tensor of t's shape, rows of whole 16-byte pieces."""
    dt = t.dtype if dtype is None else dtype
    per16 = 16 // dt.itemsize
    D = t.shape[-1]
    row = (D + per16 - 1) // per16 * per16
    o = torch.empty((*t.shape[:-1], row), dtype=dt, device=t.device)
    return o if row == D else o[..., :D]


def _on(device):
    """Launches go to the tensors' device, whichever is current."""
    return torch.cuda.device(device)


def _stream(device):
    return torch.cuda.current_stream(device).cuda_stream


def _call(device, name, *args):
    """The library's call of that name on the device's current stream, which is its last argument."""
    f = getattr(binding.lib(), name)
    if torch.cuda.current_device() == device.index:
        st = f(*args, _stream(device))
    else:
        with _on(device):
            st = f(*args, _stream(device))
    if st:
        binding._check(st, name)


# ---- rotary positions
def rope_frequencies(rot, base=10000.0, *, scaling=None, factor=1.0, trained=0.0, slow=1.0, fast=32.0, device="cuda"):
    """(freqs, amplitude) for tlin_rope: float64 [rot/2] on the device, and the factor of the rotated columns.
    scaling: None, "linear" (positions interpolated by factor), "base" (the base raised so that the slowest pair is
    interpolated by factor) or "parts" (pairs that turn more than `fast` times in `trained` positions stay, those under
    `slow` are interpolated)."""
    if scaling not in _SCALINGS:
        raise ValueError(f"scaling {scaling!r}: one of {list(_SCALINGS)} expected")
    n = int(rot)
    f, a = (ctypes.c_double * max(n // 2, 1))(), ctypes.c_double()
    st = binding.lib().tlin_rope_frequencies(n, float(base), _SCALINGS[scaling], float(factor), float(trained), float(slow),
                                             float(fast), f, ctypes.byref(a))
    binding._check(st, "tlin_rope_frequencies")
    return torch.tensor(list(f), dtype=torch.float64, device=device), a.value


def _freqs(freqs, device):
    if freqs.dtype != torch.float64 or freqs.dim() != 1 or not freqs.is_contiguous() or freqs.device != device:
        raise TypeError(f"freqs: a contiguous float64 vector on {device} expected")
    return 2 * freqs.shape[0]


def tlin_rope(x, positions, freqs, *, interleaved=False, amplitude=1.0, transpose=False, out=None):
    """Rotary positions: the first 2 * len(freqs) columns of x [B,H,rows,D] turned pair by pair, row r of batch b by
    positions[b, r] * freqs (positions int32 [rows] or [B, rows]).  transpose: the gradient of x from that of the
    result.  out: where the result goes, x itself allowed."""
    dev, dt = x.device, x.dtype
    _check(dev, dt, x=x, out=out)
    o = _like(x) if out is None else out
    if o.shape != x.shape:
        raise ValueError("out must have the shape of x")
    xs, os = _rows(x, 4, "x"), _rows(o, 4, "out")
    B, H, rows, D = x.shape
    if positions.dtype != torch.int32 or positions.device != dev:
        raise TypeError(f"positions: an int32 tensor on {dev} expected")
    if positions.shape != (rows,) and positions.shape != (B, rows):
        raise ValueError("positions are [rows] or [B, rows]")
    if rows > 1 and positions.stride(-1) != 1:
        raise ValueError("positions: rows one after another expected")
    ps = positions.stride(0) if positions.dim() == 2 and B > 1 else 0
    p = packed(TlinRopeParams, ROPE_LAYOUT, B, H, rows, D, _freqs(freqs, dev), bool(interleaved), bool(transpose), _code(dt),
               amplitude, ps, *xs, *os)
    _call(dev, "tlin_rope", p, x.data_ptr(), o.data_ptr(), positions.data_ptr(), freqs.data_ptr())
    return o


# ---- the cache
def _paged(dev, k_pages, v_pages, table, lens, starts, T, H, max_rows, dtype, out_dtype, causal, scale, strides):
    kp, vp = _rows(k_pages, 4, "k_pages"), _rows(v_pages, 4, "v_pages")
    P, HK, R, D = k_pages.shape
    if v_pages.shape != k_pages.shape:
        raise ValueError("k_pages and v_pages must have the same shape")
    S, M = _table(dev, table)
    _flat(dev, S, lens=lens)
    _flat(dev, S + 1, starts=starts)
    return packed(TlinPagedParams, PAGED_LAYOUT, S, T, H, HK, D, R, M, P, T if max_rows is None else min(int(max_rows), T), _code(dtype),
                  _code(out_dtype), bool(causal), scale, table.stride(0) if S > 1 else 0, *strides, *kp, *vp)


def _table(dev, table):
    if table.dtype != torch.int32 or table.device != dev:
        raise TypeError(f"table: an int32 tensor on {dev} expected")
    if table.dim() != 2 or (table.shape[1] > 1 and table.stride(1) != 1):
        raise ValueError("table: [sequences, pages], rows contiguous, expected")
    return table.shape


def tlin_paged_append(k, v, k_pages, v_pages, table, lens, starts, *, q=None, q_out=None, freqs=None, interleaved=False,
                      amplitude=1.0):
    """New rows k, v [HK,T,D] into the pages: rows starts[s] .. starts[s+1]-1 are the last of the lens[s] rows of
    sequence s.  With freqs (see tlin_rope) the keys are rotated by their positions on the way, and the queries q
    [H,T,D] too, into q_out (default: a new tensor; q itself allowed), which is returned."""
    dev, dt = k.device, k.dtype
    _check(dev, dt, k=k, v=v, k_pages=k_pages, v_pages=v_pages, q=q, q_out=q_out)
    HK, T, D = k.shape
    if v.shape != k.shape or k_pages.shape[1] != HK or k_pages.shape[3] != D:
        raise ValueError("k and v are [HK, T, D] with the caches' heads and columns")
    if q is None and q_out is not None:
        raise ValueError("q_out without q")
    H, qs, os = HK, (0, 0), (0, 0)
    if q is not None:
        if freqs is None:
            raise ValueError("queries are only taken to be rotated: freqs expected")
        if q.dim() != 3 or q.shape[1:] != k.shape[1:]:
            raise ValueError("q is [H, T, D] with the new rows' T and D")
        H = q.shape[0]
        if q_out is None:
            q_out = _like(q)
        if q_out.shape != q.shape:
            raise ValueError("q_out must have the shape of q")
        qs, os = _rows(q, 3, "q"), _rows(q_out, 3, "q_out")
    p = _paged(dev, k_pages, v_pages, table, lens, starts, T, H, None, dt, dt, True, 1.0,
               (*qs, *os, *_rows(k, 3, "k"), *_rows(v, 3, "v")))
    r = None
    if freqs is not None:
        r = packed(TlinRopeParams, ROPE_LAYOUT, 1, 1, 1, D, _freqs(freqs, dev), bool(interleaved), 0, 0, amplitude, 0, *(0,) * 6)
    _call(dev, "tlin_paged_append", p, r, None if q is None else q.data_ptr(), None if q is None else q_out.data_ptr(), k.data_ptr(),
          v.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), table.data_ptr(), lens.data_ptr(), starts.data_ptr(),
          None if freqs is None else freqs.data_ptr())
    return q_out


def tlin_paged_attn(q, k_pages, v_pages, table, lens, starts, *, max_rows=None, causal=True, scale=None, out_dtype=None,
                    out=None, return_lse=False, workspace=None):
    """Attention of the new rows q [H,T,D] of every sequence over its rows in the cache: causal, row i of a sequence sees
    the rows up to its own position, else all lens[s] of them.  Query head h reads key head h // (H // HK).  max_rows:
    most new rows of one sequence, where the program knows it (it picks the kernel's shape, not the result).  Returns O, or
    (O, lse) with return_lse.  Rows that belong to no sequence are not written."""
    dev, dt = q.device, q.dtype
    _check(dev, dt, q=q, k_pages=k_pages, v_pages=v_pages)
    _check(dev, out=out)
    H, T, D = q.shape
    if k_pages.shape[3] != D:
        raise ValueError("q and the caches must have the same columns")
    o = _like(q, out_dtype) if out is None else out
    if o.shape != q.shape:
        raise ValueError("out must have the shape of q")
    p = _paged(dev, k_pages, v_pages, table, lens, starts, T, H, max_rows, dt, o.dtype, causal,
               D ** -0.5 if scale is None else scale, (*_rows(q, 3, "q"), *_rows(o, 3, "out"), 0, 0, 0, 0))
    lse = torch.empty((H, T), dtype=torch.float32, device=dev) if return_lse else None
    ws, nb = _workspace(dev, workspace, binding.lib().tlin_paged_workspace_bytes(p))
    _call(dev, "tlin_paged_attn", p, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), table.data_ptr(), lens.data_ptr(),
          starts.data_ptr(), o.data_ptr(), lse.data_ptr() if return_lse else None, ws or None, nb)
    return (o, lse) if return_lse else o


def _workspace(dev, workspace, nbytes):
    from . import _default_ws, Workspace
    if workspace is None:
        key = (dev, _stream(dev))
        workspace = _default_ws.get(key)
        if workspace is None:
            workspace = _default_ws[key] = Workspace()
    return workspace.get(nbytes, dev)


# ---- pages
def _book(table, page_rows, P):
    S, M = _table(table.device, table)
    return packed(TlinBookParams, BOOK_LAYOUT, S, M, P, int(page_rows), table.stride(0) if S > 1 else 0)


def tlin_pages_free(table, lens, refs, seqs, page_rows=16):
    """The sequences in seqs (int32 [n]) give up their pages."""
    dev = table.device
    _check(dev, table=table)
    _flat(dev, 1, refs=refs)
    _flat(dev, 0, seqs=seqs)
    p = _book(table, page_rows, refs.shape[0])
    _flat(dev, p.S, lens=lens)
    _call(dev, "tlin_pages_free", p, table.data_ptr(), lens.data_ptr(), refs.data_ptr(), seqs.data_ptr(), seqs.shape[0])


def tlin_pages_fork(table, lens, refs, parents, children, page_rows):
    """Sequence children[i] becomes a copy of parents[i] that names the same pages.  Returns status int32 [n], 1 where a
    pair was passed over (see include/tlinpaged.h)."""
    dev = table.device
    _check(dev, table=table)
    _flat(dev, 1, refs=refs)
    _flat(dev, 0, parents=parents)
    _flat(dev, parents.shape[0], children=children)
    p = _book(table, page_rows, refs.shape[0])
    _flat(dev, p.S, lens=lens)
    status = torch.empty_like(parents)
    _call(dev, "tlin_pages_fork", p, table.data_ptr(), lens.data_ptr(), refs.data_ptr(), parents.data_ptr(), children.data_ptr(),
          parents.shape[0], status.data_ptr())
    return status


def tlin_pages_reserve(table, lens, refs, want, page_rows, *, workspace=None):
    """Room for want[s] more rows of every sequence; shared last pages that are not full are replaced by own ones.
    Returns (moves int32 [S, 2], count int32 [1], status int32 [S]): pairs of pages for tlin_pages_copy, and 1 where
    there was no room."""
    dev = table.device
    _check(dev, table=table)
    _flat(dev, 1, refs=refs)
    p = _book(table, page_rows, refs.shape[0])
    S = p.S
    _flat(dev, S, lens=lens, want=want)
    res = torch.empty(3 * S + 1, dtype=torch.int32, device=dev)
    at = res.data_ptr()
    ws, nb = _workspace(dev, workspace, binding.lib().tlin_pages_workspace_bytes(p))
    _call(dev, "tlin_pages_reserve", p, table.data_ptr(), lens.data_ptr(), refs.data_ptr(), want.data_ptr(), at, at + 8 * S,
          at + 8 * S + 4, ws or None, nb)
    return res[: 2 * S].view(S, 2), res[2 * S : 2 * S + 1], res[2 * S + 1 :]


def tlin_pages_compact(table, refs, *, table_out=None, refs_out=None, workspace=None):
    """Pages in use brought to the lowest ids.  Returns (table, refs, moves int32 [num_pages // 2, 2], count int32 [1]),
    table and refs in place unless table_out and refs_out are given; tlin_pages_copy moves the contents."""
    dev = table.device
    _check(dev, table=table)
    _flat(dev, 1, refs=refs)
    t = table if table_out is None else table_out
    r = refs if refs_out is None else refs_out
    P = refs.shape[0]
    p = _book(table, 16, P)
    if _table(dev, t) != table.shape or t.stride() != table.stride():
        raise ValueError("table_out must have the shape and strides of table")
    _flat(dev, P, refs_out=r)
    n = P // 2
    res = torch.empty(2 * n + 1, dtype=torch.int32, device=dev)
    at = res.data_ptr()
    ws, nb = _workspace(dev, workspace, binding.lib().tlin_pages_workspace_bytes(p))
    _call(dev, "tlin_pages_compact", p, table.data_ptr(), refs.data_ptr(), t.data_ptr(), r.data_ptr(), at, at + 8 * n, ws or None, nb)
    return t, r, res[: 2 * n].view(n, 2), res[2 * n :]


def tlin_pages_copy(k_pages, v_pages, moves, count=None):
    """Pages moves[i, 0] copied to moves[i, 1] in both caches ([num_pages, HK, page rows, D], or with a leading axis of
    layers); v_pages may be None.  count: int32 [1], how many pairs there are (default: all of moves)."""
    dev, dt = k_pages.device, k_pages.dtype
    _check(dev, dt, k_pages=k_pages, v_pages=v_pages)
    if moves.dtype != torch.int32 or moves.device != dev or moves.dim() != 2 or moves.shape[1] != 2 or not moves.is_contiguous():
        raise TypeError(f"moves: a contiguous int32 [n, 2] tensor on {dev} expected")
    if count is not None:
        _flat(dev, 1, count=count)
    axes = k_pages.dim()
    if axes not in (4, 5):
        raise ValueError("caches are [num_pages, HK, page rows, D], or with a leading axis of layers")
    st = [_rows(k_pages, axes, "k_pages"), _rows(v_pages, axes, "v_pages") if v_pages is not None else (0,) * (axes - 1)]
    if v_pages is not None and v_pages.shape != k_pages.shape:
        raise ValueError("k_pages and v_pages must have the same shape")
    L = k_pages.shape[0] if axes == 5 else 1
    P, HK, R, D = k_pages.shape[-4:]
    layer = (st[0][0], st[1][0]) if axes == 5 else (0, 0)
    p = packed(TlinCacheParams, CACHE_LAYOUT, L, P, HK, R, D, _code(dt), *layer, *st[0][-3:], *st[1][-3:])
    _call(dev, "tlin_pages_copy", p, k_pages.data_ptr(), None if v_pages is None else v_pages.data_ptr(), moves.data_ptr(),
          None if count is None else count.data_ptr(), moves.shape[0])
