"""A paged key/value cache: torch faces of the calls of include/tlinpaged.h.

Caches are ``[num_pages, key heads, page rows, D]`` tensors (any strides with whole 16-byte pieces, so a view of
``[num_pages, page rows, key heads, D]`` is one too), new rows ``[heads, T, D]`` (a view of ``[T, heads, D]`` is one), and
the table, lengths, starts and counts int32 tensors on the same device.  Nothing here synchronises.
"""
from __future__ import annotations

import ctypes
import threading

import torch

from . import binding
from .binding import BOOK_LAYOUT, CACHE_LAYOUT, PAGED_LAYOUT, ROPE_LAYOUT, TLIN_BF16, TLIN_F32

_CODES = {torch.float32: TLIN_F32, torch.bfloat16: TLIN_BF16}
_SCALINGS = {None: 0, "linear": 1, "base": 2, "parts": 3}
_I32, _F64, _BF16 = torch.int32, torch.float64, torch.bfloat16

# The calls of a step are short (a kernel takes 3 to 20 us), so the wrappers are written for few Python operations:
# parameters are packed into bytes, one comparison finds that something is wrong, and only then is it looked for what.


def _code(dtype):
    try:
        return _CODES[dtype]
    except KeyError:
        raise TypeError(f"unsupported dtype {dtype}: float32 or bfloat16 expected") from None


def _refuse(device, dtype, **tensors):
    """Says which tensor is not on the device or not of the type."""
    for name, t in tensors.items():
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError(f"{name}: libtlinattn takes device tensors only")
        if t.device != device:
            raise ValueError(f"{name} is on {t.device}, the call on {device}")
        if dtype is not None and t.dtype != dtype:
            raise TypeError(f"{name} is {t.dtype}, {dtype} expected")


def _ints(name, t, index, size):
    """An int32 vector on the device, at least `size` long."""
    if t.dtype is _I32 and t.get_device() == index and t.dim() == 1 and t.shape[0] >= size and t.is_contiguous():
        return
    if t.dtype is not _I32 or t.get_device() != index:
        raise TypeError(f"{name}: an int32 tensor on cuda:{index} expected, not {t.dtype} on {t.device}")
    raise ValueError(f"{name}: {size} entries, one after another, expected")


_whole = {}        # strides -> those of the axes before D where the library takes them for axes of any length, else False


def _rows(t, axes, name):
    """Strides of the axes before D."""
    st = t.stride()
    known = _whole.get(st)
    if known and len(known) == axes - 1:
        return known
    shape = t.shape
    if len(st) != axes or (st[-1] != 1 and shape[-1] != 1):
        raise ValueError(f"{name}: {axes} axes expected, the last one contiguous")
    if not st[-2] and shape[-2] > 1:
        raise ValueError(f"{name}: rows that lie on one another")
    if known is None:
        if len(_whole) >= 4096:
            _whole.clear()
        known = _whole[st] = st[-1] == 1 and 0 < st[-2] < 1 << 23 and not any(s % 8 for s in st[:-1]) and st[:-1]
    if known or 1 not in shape:
        return st[:-1]
    # The stride of an axis of one entry addresses nothing and may be any number: 0 stands for it, and for a row's a row of
    # whole 16-byte pieces (strides of zeros alone would be taken for those of a dense tensor).
    return (*(s if n > 1 else 0 for s, n in zip(st[:-2], shape)), st[-2] if shape[-2] > 1 else (shape[-1] + 7) // 8 * 8)


def _table_stride(table, S):
    st = table.stride(0) if S > 1 else 0
    if S > 1 and not st:
        raise ValueError("table: rows that lie on one another")
    return st


def _table_like(t, table):
    return t.shape == table.shape and (t.shape[0] == 1 or t.stride(0) == table.stride(0))


def _like(t, dtype=None):
    """An uninitialised tensor of t's shape, rows of whole 16-byte pieces (and in t's order, where t is dense)."""
    dt = t.dtype if dtype is None else dtype
    shape = t.shape
    D = shape[-1]
    row = (D + 7) // 8 * 8 if dt is _BF16 else (D + 3) // 4 * 4
    if row == D:
        return torch.empty_like(t, dtype=dt)
    return torch.empty((*shape[:-1], row), dtype=dt, device=t.device)[..., :D]


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
_calls = None


def _library():
    """The library with its parameter structures as bytes."""
    global _calls
    if _calls is None:
        binding.lib()           # (raises if it is not built)
        L = ctypes.CDLL(binding.LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        for name, res, args in (
                ("tlin_rope", ctypes.c_int, [vp] * 6), ("tlin_paged_append", ctypes.c_int, [vp] * 13),
                ("tlin_paged_workspace_bytes", sz, [vp]), ("tlin_paged_attn", ctypes.c_int, [vp] * 10 + [sz, vp]),
                ("tlin_pages_free", ctypes.c_int, [vp] * 5 + [i32, vp]), ("tlin_pages_fork", ctypes.c_int, [vp] * 6 + [i32, vp, vp]),
                ("tlin_pages_workspace_bytes", sz, [vp]), ("tlin_pages_reserve", ctypes.c_int, [vp] * 9 + [sz, vp]),
                ("tlin_pages_compact", ctypes.c_int, [vp] * 8 + [sz, vp]), ("tlin_pages_copy", ctypes.c_int, [vp] * 5 + [i32, vp])):
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _calls = L
    return _calls


def _call(index, stream, name, *args):
    """The library's call of that name, launched on the tensors' device whichever is current."""
    f = getattr(_calls or _library(), name)
    if torch._C._cuda_getDevice() == index:
        st = f(*args, stream)
    else:
        with torch.cuda.device(index):
            st = f(*args, stream)
    if st:
        binding._check(st, name)


_ws_bytes = {}     # what the library answered, by the sizes that it goes by


class _Scratch(threading.local):
    def __init__(self):
        self.of = {}     # (device, stream) -> (aligned address, bytes behind it, buffer)


_scratch = _Scratch()


def _workspace(device, index, stream, workspace, nbytes):
    """Device scratch, (address, bytes, what keeps it): the caller's, or one kept per host thread, device and stream and grown
    on demand.  Not per stream alone: calls of two threads on one stream may enqueue their launches in turn, and a call's
    launches hand their results to each other here.  A call that is captured gets scratch of its own from the graph's memory:
    graphs captured on one stream may be replayed on two, and what is kept here may be replaced by a larger one."""
    if workspace is not None:
        return (*workspace.get(nbytes, device), None)
    have = _scratch.of.get((index, stream))
    if torch._C._cuda_getDevice() == index:
        capturing = torch._C._cuda_isCurrentStreamCapturing()
    else:
        with torch.cuda.device(index):
            capturing = torch._C._cuda_isCurrentStreamCapturing()
    if have is None or have[1] < nbytes or capturing:
        buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        have = ((buf.data_ptr() + 255) // 256 * 256, nbytes, buf)
        if not capturing:
            _scratch.of[(index, stream)] = have
    return have


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


def _freqs(freqs, index):
    if freqs.dtype is not _F64 or freqs.dim() != 1 or freqs.get_device() != index or not freqs.is_contiguous():
        raise TypeError(f"freqs: a contiguous float64 vector on cuda:{index} expected")
    return 2 * freqs.shape[0]


def tlin_rope(x, positions, freqs, *, interleaved=False, amplitude=1.0, transpose=False, out=None):
    """Rotary positions: the first 2 * len(freqs) columns of x [B,H,rows,D] turned pair by pair, row r of batch b by
    positions[b, r] * freqs (positions int32 [rows] or [B, rows]).  transpose: the gradient of x from that of the
    result.  out: where the result goes, x itself allowed."""
    dt, index = x.dtype, x.get_device()
    if index < 0 or (out is not None and (out.get_device() != index or out.dtype is not dt)):
        _refuse(x.device, dt, x=x, out=out)
    code = _code(dt)
    o = _like(x) if out is None else out
    if o.shape != x.shape:
        raise ValueError("out must have the shape of x")
    xs, os = _rows(x, 4, "x"), _rows(o, 4, "out")
    B, H, rows, D = x.shape
    if positions.dtype is not _I32 or positions.get_device() != index:
        raise TypeError(f"positions: an int32 tensor on cuda:{index} expected")
    ps = positions.shape
    if ps != (rows,) and ps != (B, rows):
        raise ValueError("positions are [rows] or [B, rows]")
    if rows > 1 and positions.stride(-1) != 1:
        raise ValueError("positions: rows one after another expected")
    p = ROPE_LAYOUT.pack(B, H, rows, D, _freqs(freqs, index), bool(interleaved), bool(transpose), code, amplitude,
                         positions.stride(0) if len(ps) == 2 and B > 1 else 0, *xs, *os)
    _call(index, _raw_stream(index), "tlin_rope", p, x.data_ptr(), o.data_ptr(), positions.data_ptr(), freqs.data_ptr())
    return o


# ---- the cache
def _table(index, table):
    if table.dtype is not _I32 or table.get_device() != index:
        raise TypeError(f"table: an int32 tensor on cuda:{index} expected")
    shape = table.shape
    if len(shape) != 2 or (shape[1] > 1 and table.stride(1) != 1):
        raise ValueError("table: [sequences, pages], rows contiguous, expected")
    return shape


def _paged(index, k_pages, v_pages, table, lens, starts, T, H, max_rows, code, out_code, causal, scale, strides):
    kp, vp, shape, entries = k_pages.stride(), v_pages.stride(), k_pages.shape, table.shape
    if len(kp) != 4 or v_pages.shape != shape or kp[3] != 1 or vp[3] != 1 or not (kp[2] and vp[2]):
        _rows(k_pages, 4, "k_pages"), _rows(v_pages, 4, "v_pages")
        raise ValueError("k_pages and v_pages must have the same shape")
    P, HK, R, D = shape
    if P == 1 or HK == 1:           # (strides that may be any number)
        kp, vp = _rows(k_pages, 4, "k_pages"), _rows(v_pages, 4, "v_pages")
    if table.dtype is not _I32 or table.get_device() != index or len(entries) != 2 or (entries[1] > 1 and table.stride(1) != 1):
        _table(index, table)
    S, M = entries
    _ints("lens", lens, index, S)
    _ints("starts", starts, index, S + 1)
    return PAGED_LAYOUT.pack(S, T, H, HK, D, R, M, P, T if max_rows is None else min(int(max_rows), T), code, out_code, bool(causal),
                             scale, _table_stride(table, S), *strides, kp[0], kp[1], kp[2], vp[0], vp[1], vp[2])


def tlin_paged_append(k, v, k_pages, v_pages, table, lens, starts, *, q=None, q_out=None, freqs=None, interleaved=False,
                      amplitude=1.0):
    """New rows k, v [HK,T,D] into the pages: rows starts[s] .. starts[s+1]-1 are the last of the lens[s] rows of
    sequence s.  With freqs (see tlin_rope) the keys are rotated by their positions on the way, and the queries q
    [H,T,D] too, into q_out (default: a new tensor; q itself allowed), which is returned."""
    dt, index = k.dtype, k.get_device()
    if not (index >= 0 and v.get_device() == k_pages.get_device() == v_pages.get_device() == index and v.dtype is dt
            and k_pages.dtype is dt and v_pages.dtype is dt):
        _refuse(k.device, dt, k=k, v=v, k_pages=k_pages, v_pages=v_pages)
    code = _code(dt)
    shape = k.shape
    if len(shape) != 3 or v.shape != shape or k_pages.dim() != 4 or k_pages.shape[1] != shape[0] or k_pages.shape[3] != shape[2]:
        raise ValueError("k and v are [HK, T, D] with the caches' heads and columns")
    HK, T, D = shape
    if q is None and q_out is not None:
        raise ValueError("q_out without q")
    H, strides, qa, oa = HK, (0, 0, 0, 0), None, None
    if q is not None:
        if freqs is None:
            raise ValueError("queries are only taken to be rotated: freqs expected")
        if q.dim() != 3 or q.shape[1:] != shape[1:]:
            raise ValueError("q is [H, T, D] with the new rows' T and D")
        if q_out is None:
            q_out = _like(q)
        if not (q.get_device() == q_out.get_device() == index and q.dtype is dt and q_out.dtype is dt):
            _refuse(k.device, dt, q=q, q_out=q_out)
        if q_out.shape != q.shape:
            raise ValueError("q_out must have the shape of q")
        H, qa, oa = q.shape[0], q.data_ptr(), q_out.data_ptr()
        strides = (*_rows(q, 3, "q"), *_rows(q_out, 3, "q_out"))
    p = _paged(index, k_pages, v_pages, table, lens, starts, T, H, None, code, code, True, 1.0,
               (*strides, *_rows(k, 3, "k"), *_rows(v, 3, "v")))
    r = fa = None
    if freqs is not None:
        r = ROPE_LAYOUT.pack(1, 1, 1, D, _freqs(freqs, index), bool(interleaved), 0, 0, amplitude, 0, 0, 0, 0, 0, 0, 0)
        fa = freqs.data_ptr()
    _call(index, _raw_stream(index), "tlin_paged_append", p, r, qa, oa, k.data_ptr(), v.data_ptr(), k_pages.data_ptr(),
          v_pages.data_ptr(), table.data_ptr(), lens.data_ptr(), starts.data_ptr(), fa)
    return q_out


def tlin_paged_attn(q, k_pages, v_pages, table, lens, starts, *, max_rows=None, causal=True, scale=None, out_dtype=None,
                    out=None, return_lse=False, workspace=None):
    """Attention of the new rows q [H,T,D] of every sequence over its rows in the cache: causal, row i of a sequence sees
    the rows up to its own position, else all lens[s] of them.  Query head h reads key head h // (H // HK).  max_rows:
    most new rows of one sequence (it picks the kernel's shape, not the result).  Give it wherever the program knows it: without it
    all T rows are taken for one sequence's, and a step of many single rows runs in workgroups of up to 256 rows that it leaves
    almost empty.  Returns O, or (O, lse) with return_lse.  Rows that belong to no sequence are not written.  bf16 caches: weights
    are rounded to bf16 for the value product, whatever out_dtype is (sums and log-sum-exp are fp32)."""
    dt, index, device = q.dtype, q.get_device(), q.device
    if not (index >= 0 and k_pages.get_device() == v_pages.get_device() == index and k_pages.dtype is dt and v_pages.dtype is dt
            and (out is None or out.get_device() == index)):
        _refuse(device, dt, q=q, k_pages=k_pages, v_pages=v_pages)
        _refuse(device, None, out=out)
    code = _code(dt)
    if q.dim() != 3 or k_pages.dim() != 4 or k_pages.shape[3] != q.shape[2]:
        raise ValueError("q is [H, T, D] with the caches' columns")
    H, T, D = q.shape
    o = _like(q, out_dtype) if out is None else out
    if o.shape != q.shape:
        raise ValueError("out must have the shape of q")
    p = _paged(index, k_pages, v_pages, table, lens, starts, T, H, max_rows, code, _code(o.dtype), causal,
               D ** -0.5 if scale is None else scale, (*_rows(q, 3, "q"), *_rows(o, 3, "out"), 0, 0, 0, 0))
    lse = torch.empty((H, T), dtype=torch.float32, device=device) if return_lse else None
    stream = _raw_stream(index)
    key = (H, k_pages.shape[1], D, code, T if max_rows is None else max_rows if max_rows < T else T)
    need = _ws_bytes.get(key)
    if need is None:
        need = (_calls or _library()).tlin_paged_workspace_bytes(p)
        if need:
            _ws_bytes[key] = need
    ws, nb, _kept = _workspace(device, index, stream, workspace, need)
    _call(index, stream, "tlin_paged_attn", p, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), table.data_ptr(), lens.data_ptr(),
          starts.data_ptr(), o.data_ptr(), lse.data_ptr() if return_lse else None, ws or None, nb)
    return (o, lse) if return_lse else o


# ---- pages
def _book(table, refs, page_rows):
    """(parameters, sequences, device index) of a book, its table and counts checked."""
    index = table.get_device()
    if index < 0:
        _refuse(table.device, None, table=table)
    S, M = _table(index, table)
    _ints("refs", refs, index, 1)
    return BOOK_LAYOUT.pack(S, M, refs.shape[0], int(page_rows), _table_stride(table, S)), S, index


def tlin_pages_free(table, lens, refs, seqs, page_rows=16):
    """The sequences in seqs (int32 [n]) give up their pages."""
    p, S, index = _book(table, refs, page_rows)
    _ints("lens", lens, index, S)
    _ints("seqs", seqs, index, 0)
    _call(index, _raw_stream(index), "tlin_pages_free", p, table.data_ptr(), lens.data_ptr(), refs.data_ptr(), seqs.data_ptr(),
          seqs.shape[0])


def tlin_pages_fork(table, lens, refs, parents, children, page_rows):
    """Sequence children[i] becomes a copy of parents[i] that names the same pages.  Returns status int32 [n], 1 where a
    pair was passed over (see include/tlinpaged.h)."""
    p, S, index = _book(table, refs, page_rows)
    _ints("lens", lens, index, S)
    _ints("parents", parents, index, 0)
    n = parents.shape[0]
    _ints("children", children, index, n)
    status = torch.empty_like(parents)
    _call(index, _raw_stream(index), "tlin_pages_fork", p, table.data_ptr(), lens.data_ptr(), refs.data_ptr(), parents.data_ptr(),
          children.data_ptr(), n, status.data_ptr())
    return status


def _pages_workspace(table, index, stream, workspace, p):
    return _workspace(table.device, index, stream, workspace, (_calls or _library()).tlin_pages_workspace_bytes(p))


def tlin_pages_reserve(table, lens, refs, want, page_rows, *, workspace=None):
    """Room for want[s] more rows of every sequence; shared last pages that are not full are replaced by own ones.
    Returns (moves int32 [S, 2], count int32 [1], status int32 [S]): pairs of pages for tlin_pages_copy, and 1 where
    there was no room."""
    p, S, index = _book(table, refs, page_rows)
    _ints("lens", lens, index, S)
    _ints("want", want, index, S)
    res = torch.empty(3 * S + 1, dtype=_I32, device=table.device)
    at, stream = res.data_ptr(), _raw_stream(index)
    ws, nb, _kept = _pages_workspace(table, index, stream, workspace, p)
    _call(index, stream, "tlin_pages_reserve", p, table.data_ptr(), lens.data_ptr(), refs.data_ptr(), want.data_ptr(), at, at + 8 * S,
          at + 8 * S + 4, ws or None, nb)
    return res.as_strided((S, 2), (2, 1), 0), res.as_strided((1,), (1,), 2 * S), res.as_strided((S,), (1,), 2 * S + 1)


def tlin_pages_compact(table, refs, *, table_out=None, refs_out=None, workspace=None):
    """Pages in use brought to the lowest ids.  Returns (table, refs, moves int32 [num_pages // 2, 2], count int32 [1]),
    table and refs in place unless table_out and refs_out are given; tlin_pages_copy moves the contents."""
    p, _, index = _book(table, refs, 16)
    t = table if table_out is None else table_out
    r = refs if refs_out is None else refs_out
    P = refs.shape[0]
    _table(index, t)
    if not _table_like(t, table):
        raise ValueError("table_out must have the shape and strides of table")
    _ints("refs_out", r, index, P)
    n = P // 2
    res = torch.empty(2 * n + 1, dtype=_I32, device=table.device)
    at, stream = res.data_ptr(), _raw_stream(index)
    ws, nb, _kept = _pages_workspace(table, index, stream, workspace, p)
    _call(index, stream, "tlin_pages_compact", p, table.data_ptr(), refs.data_ptr(), t.data_ptr(), r.data_ptr(), at, at + 8 * n, ws or None,
          nb)
    return t, r, res.as_strided((n, 2), (2, 1), 0), res.as_strided((1,), (1,), 2 * n)


def tlin_pages_copy(k_pages, v_pages, moves, count=None):
    """Pages moves[i, 0] copied to moves[i, 1] in both caches ([num_pages, HK, page rows, D], or with a leading axis of
    layers); v_pages may be None.  count: int32 [1], how many pairs there are (default: all of moves)."""
    dt, index = k_pages.dtype, k_pages.get_device()
    if index < 0 or (v_pages is not None and (v_pages.get_device() != index or v_pages.dtype is not dt)):
        _refuse(k_pages.device, dt, k_pages=k_pages, v_pages=v_pages)
    if moves.dtype is not _I32 or moves.get_device() != index or moves.dim() != 2 or moves.shape[1] != 2 or not moves.is_contiguous():
        raise TypeError(f"moves: a contiguous int32 [n, 2] tensor on cuda:{index} expected")
    if count is not None:
        _ints("count", count, index, 1)
    shape = k_pages.shape
    axes = len(shape)
    if axes not in (4, 5):
        raise ValueError("caches are [num_pages, HK, page rows, D], or with a leading axis of layers")
    if v_pages is not None and v_pages.shape != shape:
        raise ValueError("k_pages and v_pages must have the same shape")
    ks = _rows(k_pages, axes, "k_pages")
    vs = _rows(v_pages, axes, "v_pages") if v_pages is not None else (0,) * (axes - 1)
    L, kl, vl = (shape[0], ks[0], vs[0]) if axes == 5 else (1, 0, 0)
    if L > 1 and not (kl and (vl or v_pages is None)):
        raise ValueError("layers that lie on one another")
    p = CACHE_LAYOUT.pack(L, *shape[-4:], _code(dt), kl, vl, *ks[-3:], *vs[-3:])
    _call(index, _raw_stream(index), "tlin_pages_copy", p, k_pages.data_ptr(), None if v_pages is None else v_pages.data_ptr(),
          moves.data_ptr(), None if count is None else count.data_ptr(), moves.shape[0])
