"""ctypes marshalling for the rotary positions and the 8-bit key/value cache of
include/rollout.h.  No computation happens here."""
from __future__ import annotations

import ctypes as C
import struct
from typing import NamedTuple, Optional

from . import _lib
from ._lib import _check, _dev, _gpu, load_library

ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {None: 0, "linear": 1, "base": 2, "bands": 3}
_MOST = 2 ** 31 - 1     # sizes are int32 in the library; or-ed together, all are at most this or the result is more


class rg_kv8_cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("pages", C.c_int64), ("n_kv", C.c_int32), ("head_dim", C.c_int32), ("page_tokens", C.c_int32)]


class rg_kv8_batch(C.Structure):
    _fields_ = [("page_tab", C.c_void_p), ("tab_rows", C.c_int32), ("tab_stride", C.c_int32), ("tab_row", C.c_void_p),
                ("seq_off", C.c_void_p), ("seq_len", C.c_void_p), ("n_seqs", C.c_int32), ("rows", C.c_int32)]


# The same two as bytes: a call that passes in few questions packs them in a
# fraction of the time that filling a ctypes structure takes.
_CACHE, _BATCH = struct.Struct("@4Pq3i4x").pack, struct.Struct("@P2i3P2i").pack

_P, _I, _L, _D = C.c_void_p, C.c_int32, C.c_int64, C.c_double
_ARGS = {
    "rg_rope_table": ([_P, _P, _I, _I, _D, _I, _D, _D, _D, _D, _P], C.c_int),
    "rg_rope": ([_I, _P, _L, _L, _P, _L, _L, _P, _I, _I, _I, _P, _P, _I, _I, _I, _I, _P], C.c_int),
    "rg_kv8_append": ([_P, _P, _I, _P, _L, _L, _P, _L, _L, _P, _L, _L, _P, _L, _L,
                       _I, _P, _P, _I, _I, _I, _P], C.c_int),
    "rg_kv8_attention_scratch": ([_I, _I, _I, _I, _I, _I, _I], C.c_int64),
    "rg_kv8_attention": ([_P, _P, _I, _P, _L, _L, _I, _P, C.c_float, _I, _P, _L, _P],
                         C.c_int),
}
_ready = None
_BF16 = _F32 = _E4M3 = _I32 = _device = _raw_stream = _empty_like = _grad_on = _recorded = None


def _library():
    global _ready, _BF16, _F32, _E4M3, _I32, _device, _raw_stream, _empty_like, _grad_on, _recorded
    if _ready is None:
        lib = load_library()
        for name, (args, res) in _ARGS.items():
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = args, res
        import torch
        _BF16, _F32, _E4M3, _I32 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.int32
        _device, _raw_stream, _empty_like = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream, torch.empty_like
        _grad_on, _recorded = torch.is_grad_enabled, _recorded_rope()
        _ready = lib
    return _ready


# A decode step's calls take a few microseconds on the device, and naming what is
# wrong with an argument takes longer than that to set up.  So each call first asks
# whether everything is as it should be, in the fewest questions; only where that
# fails does it go through the checks that say what and raise, or find nothing
# wrong (another device, a given stream) and go on.  What is no tensor answers the
# questions with an AttributeError, which is a no.
def _cache_fits(cache, dev):
    """(rg_kv8_cache as bytes, n_kv, head_dim, page_tokens) of a cache whose tensors are all in place, or None."""
    k, v, ks, vs = cache
    if not (k.dtype is v.dtype is _E4M3 and ks.dtype is vs.dtype is _F32 and
            k.get_device() == v.get_device() == ks.get_device() == vs.get_device() == dev and
            k.is_contiguous() and v.is_contiguous() and ks.is_contiguous() and vs.is_contiguous()):
        return None
    shape, scales = k.shape, ks.shape
    if len(shape) != 4 or v.shape != shape or vs.shape != scales:
        return None
    pages, n_kv, parts, n = shape
    if n % 16 or scales != (pages, n_kv, parts):
        return None
    hd, page = n // 16, 16 * parts
    return _CACHE(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), pages, n_kv, hd, page), n_kv, hd, page


def _batch_fits(rows, page_tab, seq_len, seq_off, tab_row, dev):
    """(rg_kv8_batch as bytes, sequences, pages of a table row) where a batch's tensors are all in place, or None."""
    if not (page_tab.dtype is seq_len.dtype is _I32 and page_tab.get_device() == seq_len.get_device() == dev and
            page_tab.is_contiguous() and seq_len.is_contiguous() and page_tab.dim() == 2 and seq_len.dim() == 1):
        return None
    n = seq_len.shape[0]
    tab_rows, stride = page_tab.shape
    if rows | n | tab_rows | stride > _MOST:
        return None
    off = row = 0
    if seq_off is not None:
        if not (seq_off.dtype is _I32 and seq_off.get_device() == dev and seq_off.is_contiguous() and
                seq_off.shape == (n + 1,)):
            return None
        off = seq_off.data_ptr()
    elif n != rows:
        return None
    if tab_row is not None:
        if not (tab_row.dtype is _I32 and tab_row.get_device() == dev and tab_row.is_contiguous() and tab_row.shape == (n,)):
            return None
        row = tab_row.data_ptr()
    elif tab_rows < n:
        return None
    return _BATCH(page_tab.data_ptr(), tab_rows, stride, row, off, seq_len.data_ptr(), n, rows), n, stride


def _table_fits(cos, sin, hd, dev):
    """(turned dims, positions) of a rotary table that is in place, or None."""
    if not (cos.dtype is sin.dtype is _F32 and cos.get_device() == sin.get_device() == dev and cos.is_contiguous() and
            sin.is_contiguous()):
        return None
    shape = cos.shape
    if len(shape) != 2 or sin.shape != shape:
        return None
    n, pairs = shape
    return (2 * pairs, n) if 1 <= n <= _MOST and 2 <= 2 * pairs <= hd else None


def _dense(like, shape):
    """A contiguous tensor of like's type and device."""
    return _empty_like(like) if like.is_contiguous() else like.new_empty(shape)


class _On:
    """The device of the call's tensors as the current one, where it is another."""

    def __init__(self, device):
        import torch
        self.ctx = None
        if device.index != torch.cuda.current_device():
            self.ctx = torch.cuda.device(device)

    def __enter__(self):
        if self.ctx is not None:
            self.ctx.__enter__()

    def __exit__(self, *exc):
        if self.ctx is not None:
            self.ctx.__exit__(*exc)


def _stream(device, stream) -> int:
    import torch
    return int(stream.cuda_stream) if stream is not None else torch._C._cuda_getCurrentRawStream(device.index)


def _empty(like, shape, dtype, stream):
    """Memory whose next owner waits for this call's work: the caching allocator
    orders a block's uses by the stream that was current when it was made."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=like.device)


def _sizes(**sizes):
    for name, n in sizes.items():
        if n > _MOST:
            raise ValueError(f"{name} must be below 2^31, got {n}")


def _view(name, t, dtype, shape):
    """A [rows, heads, head_dim] view: any strides between rows and heads, dims adjacent."""
    import torch
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor, got {type(t).__name__}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.stride(2) != 1 and t.shape[2] != 1:
        raise ValueError(f"{name} must have its last dimension contiguous")
    return t


def _written(name, t):
    """An output view must not put two of its elements in one place."""
    r, h, d = t.shape
    a, b = t.stride(0), t.stride(1)
    ok = (b >= d or h <= 1) and (a >= (h - 1) * b + d or r <= 1)
    if not ok and not ((a >= d or r <= 1) and (b >= (r - 1) * a + d or h <= 1)):
        raise ValueError(f"{name} has overlapping rows or heads (strides {tuple(t.stride())})")
    return t


def _one_device(tensors):
    _gpu(**tensors)
    devices = {t.device for t in tensors.values() if t is not None}
    if len(devices) > 1:
        raise TypeError("tensors must be on one device, got " + ", ".join(sorted(str(d) for d in devices)))


def _float_type(name, t):
    import torch
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor, got {type(t).__name__}")
    if t.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"{name} must have dtype torch.bfloat16 or torch.float32, got {t.dtype}")
    if t.dim() != 3:
        raise ValueError(f"{name} must have 3 dimensions [rows, heads, head_dim], got shape {tuple(t.shape)}")
    return t.dtype, 1 if t.dtype == torch.bfloat16 else 0


def _tables(cos, sin, head_dim, layout):
    """Checks a rotary table; returns the turned dims."""
    import torch
    if layout not in ROPE_LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(ROPE_LAYOUTS)}")
    _dev("cos", cos, torch.float32, ndim=2)
    _dev("sin", sin, torch.float32, tuple(cos.shape))
    rot = 2 * int(cos.shape[1])
    _sizes(positions=cos.shape[0])
    if cos.shape[0] < 1 or not 2 <= rot <= head_dim:
        raise ValueError(f"a table of {tuple(cos.shape)} does not fit head_dim {head_dim}")
    return rot


def rope_table(n_pos: int, rot_dim: int, theta: float = 1e4, scaling: Optional[str] = None, factor: float = 1.0,
               length: float = 0.0, slow: float = 1.0, fast: float = 32.0, device="cuda", stream=None):
    """(cos, sin) of positions 0 .. n_pos-1: device fp32 [n_pos, rot_dim/2].
    ``scaling``: None, "linear", "base" or "bands" with ``factor`` (and for
    "bands" the trained ``length``); see rg_rope_table in rollout.h."""
    import torch
    lib = _ready or _library()
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"scaling must be one of {list(ROPE_SCALINGS)}")
    n_pos, rot_dim = int(n_pos), int(rot_dim)
    if n_pos < 1 or rot_dim < 2 or rot_dim % 2:
        raise ValueError(f"need n_pos >= 1 and an even rot_dim >= 2, got {n_pos} and {rot_dim}")
    _sizes(n_pos=n_pos, rot_dim=rot_dim)
    device = torch.device(device)
    if device.type != "cuda":
        raise TypeError(f"tables are made in GPU memory, got device {device}")
    if device.index is None:
        device = torch.device("cuda", torch.cuda.current_device())
    with _On(device):
        like = torch.empty(0, device=device)
        cos = _empty(like, (n_pos, rot_dim // 2), torch.float32, stream)
        sin = _empty(like, (n_pos, rot_dim // 2), torch.float32, stream)
        _check(lib.rg_rope_table(cos.data_ptr(), sin.data_ptr(), n_pos, rot_dim, float(theta), ROPE_SCALINGS[scaling],
                                 float(factor), float(length), float(slow), float(fast), _stream(device, stream)))
    return cos, sin


def _recorded_rope():
    """rope as a node of an autograd graph: its gradient is the turn the other way."""
    import torch

    class Rope(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, pos, cos, sin, layout, inverse, stream):
            ctx.save_for_backward(pos, cos, sin)
            ctx.turn = layout, inverse
            return rope(x, pos, cos, sin, layout, inverse, stream=stream)   # grad mode is off here

        @staticmethod
        def backward(ctx, g):
            layout, inverse = ctx.turn
            g = g if g.stride(2) == 1 else g.contiguous()                   # one value expanded, as sum() gives
            return rope(g, *ctx.saved_tensors, layout, not inverse), None, None, None, None, None, None

    return Rope.apply


def _rope_now(lib, x, pos, cos, sin, layout, inverse):
    """The call where every argument is in place, else None."""
    if (x.requires_grad or cos.requires_grad or sin.requires_grad) and _grad_on():
        return None
    dt, dev = x.dtype, x.get_device()
    if not ((dt is _BF16 or dt is _F32) and dev >= 0 and _device() == dev and layout in ROPE_LAYOUTS and x.dim() == 3):
        return None
    rows, heads, hd = x.shape
    a, b, one = x.stride()
    t = _table_fits(cos, sin, hd, dev)
    if not (t is not None and one == 1 and hd % 2 == 0 and rows | heads | hd <= _MOST and pos.dtype is _I32 and
            pos.get_device() == dev and pos.is_contiguous() and pos.shape == (rows,)):
        return None
    rot, n_pos = t
    y = _dense(x, (rows, heads, hd))
    rc = lib.rg_rope(1 if dt is _BF16 else 0, x.data_ptr(), a, b, y.data_ptr(), heads * hd, hd, pos.data_ptr(), rows,
                     heads, hd, cos.data_ptr(), sin.data_ptr(), n_pos, rot, ROPE_LAYOUTS[layout], 1 if inverse else 0,
                     _raw_stream(dev))
    if rc:
        _check(rc)
    return y


def rope(x, pos, cos, sin, layout: str = "half", inverse: bool = False, out=None, stream=None):
    """Turns the heads of x (bf16 or fp32 [rows, heads, head_dim], rows and heads
    at any strides) by their rows' positions pos (int32 [rows]); cos and sin are
    a rope_table of at most head_dim dims.  ``inverse=True`` turns back: the
    gradient with respect to x, given the one with respect to the result.  An x
    that requires a gradient is recorded so by autograd (without ``out``; the
    table takes no gradient).
    ``out`` may be x.  See rg_rope in rollout.h."""
    lib = _ready or _library()
    if out is None and stream is None:
        try:
            y = _rope_now(lib, x, pos, cos, sin, layout, inverse)
        except AttributeError:
            y = None
        if y is not None:
            return y
    dt, code = _float_type("x", x)
    rows, heads, hd = x.shape
    _view("x", x, dt, x.shape)
    _sizes(rows=rows, heads=heads, head_dim=hd)
    if hd < 2 or hd % 2:
        raise ValueError(f"head_dim must be even, got {hd}")
    rot = _tables(cos, sin, hd, layout)
    _dev("pos", pos, _I32, (rows,))
    if out is not None:
        _written("out", _view("out", out, dt, x.shape))
    if _grad_on():
        if cos.requires_grad or sin.requires_grad:
            raise ValueError("cos and sin take no gradient: detach them")
        if out is not None and (x.requires_grad or out.requires_grad):
            raise ValueError("with out the call is not recorded and a gradient would be lost: leave it out, or detach x and out")
        if x.requires_grad:
            return _recorded(x, pos, cos, sin, layout, inverse, stream)
    _one_device(dict(x=x, pos=pos, cos=cos, sin=sin, out=out))
    dev = x.device
    with _On(dev):
        y = _empty(x, (rows, heads, hd), dt, stream) if out is None else out
        _check(lib.rg_rope(code, x.data_ptr(), x.stride(0), x.stride(1), y.data_ptr(), y.stride(0), y.stride(1),
                           pos.data_ptr(), rows, heads, hd, cos.data_ptr(), sin.data_ptr(), cos.shape[0], rot,
                           ROPE_LAYOUTS[layout], 1 if inverse else 0, _stream(dev, stream)))
    return y


class Kv8Cache(NamedTuple):
    """The tensors of a paged e4m3 cache (rg_kv8_cache in rollout.h): codes
    float8_e4m3fn [pages, n_kv, page_tokens/16, 16*head_dim] and scales fp32
    [pages, n_kv, page_tokens/16].  The caller's own memory: pages are handed
    out, shared, copied and saved as the program likes."""
    k: object
    v: object
    k_scale: object
    v_scale: object

    @classmethod
    def empty(cls, pages: int, n_kv: int, head_dim: int, page_tokens: int = 16, device="cuda"):
        """A cache whose pages hold nothing yet (contents undefined)."""
        import torch
        if page_tokens not in (16, 32, 64, 128, 256, 512, 1024):
            raise ValueError(f"page_tokens must be a multiple of 16 by a power of two, at most 1024, got {page_tokens}")
        if head_dim not in (64, 128):
            raise ValueError(f"head_dim must be 64 or 128, got {head_dim}")
        shape = (pages, n_kv, page_tokens // 16)
        k, v = (torch.empty(*shape, 16 * head_dim, dtype=torch.float8_e4m3fn, device=device) for _ in range(2))
        ks, vs = (torch.empty(shape, dtype=torch.float32, device=device) for _ in range(2))
        return cls(k, v, ks, vs)


def _cache_args(cache):
    import torch
    k, v, ks, vs = cache
    _dev("cache.k", k, torch.float8_e4m3fn, ndim=4)
    shape = k.shape
    _dev("cache.v", v, torch.float8_e4m3fn, shape)
    _dev("cache.k_scale", ks, torch.float32, shape[:3])
    _dev("cache.v_scale", vs, torch.float32, shape[:3])
    pages, n_kv, parts, n = shape
    if n % 16:
        raise ValueError(f"cache.k must have blocks of 16 * head_dim codes, got shape {tuple(shape)}")
    return rg_kv8_cache(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), pages, n_kv, n // 16, 16 * parts)


def _batch_args(rows, page_tab, seq_len, seq_off, tab_row):
    import torch
    _dev("page_tab", page_tab, torch.int32, ndim=2)
    _dev("seq_len", seq_len, torch.int32, ndim=1)
    n = seq_len.shape[0]
    _sizes(rows=rows, sequences=n, **{"page_tab's rows": page_tab.shape[0], "page_tab's pages": page_tab.shape[1]})
    if seq_off is not None:
        _dev("seq_off", seq_off, torch.int32, (n + 1,))
    elif n != rows:
        raise ValueError(f"without seq_off there is one row a sequence: {rows} rows, {n} sequences")
    if tab_row is not None:
        _dev("tab_row", tab_row, torch.int32, (n,))
    elif page_tab.shape[0] < n:
        raise ValueError(f"page_tab must have a row for each of {n} sequences, got {page_tab.shape[0]}")
    return rg_kv8_batch(page_tab.data_ptr(), page_tab.shape[0], page_tab.shape[1],
                        0 if tab_row is None else tab_row.data_ptr(), 0 if seq_off is None else seq_off.data_ptr(),
                        seq_len.data_ptr(), n, rows)


def _append_now(lib, cache, k, v, page_tab, seq_len, seq_off, q, cos, sin, layout, tab_row):
    """(True, the result) of the call where every argument is in place, else (False, None)."""
    no = False, None
    dt, dev = k.dtype, k.get_device()
    if not ((dt is _BF16 or dt is _F32) and dev >= 0 and _device() == dev and k.dim() == 3 and layout in ROPE_LAYOUTS):
        return no
    rows = k.shape[0]
    c = _cache_fits(cache, dev)
    b = _batch_fits(rows, page_tab, seq_len, seq_off, tab_row, dev)
    if c is None or b is None:
        return no
    c, n_kv, hd, _ = c
    shape = rows, n_kv, hd
    kr, kh, k1 = k.stride()
    if not (k.shape == shape and v.dtype is dt and v.get_device() == dev and v.shape == shape and k1 == 1):
        return no
    vr, vh, v1 = v.stride()
    if v1 != 1:
        return no
    rot = n_pos = cp = sp = 0
    if cos is not None:
        t = _table_fits(cos, sin, hd, dev)
        if t is None:
            return no
        rot, n_pos = t
        cp, sp = cos.data_ptr(), sin.data_ptr()
    elif sin is not None:
        return no
    y, n_q, qp, qr, qh, yp = None, 0, 0, 0, 0, 0
    if q is not None:
        if not (q.dtype is dt and q.get_device() == dev and q.dim() == 3):
            return no
        q0, n_q, qd = q.shape
        qr, qh, q1 = q.stride()
        if not (q0 == rows and qd == hd and q1 == 1 and 0 < n_q <= _MOST and n_q % n_kv == 0):
            return no
        y = _dense(q, (rows, n_q, hd))
        qp, yp = q.data_ptr(), y.data_ptr()
    rc = lib.rg_kv8_append(c, b[0], 1 if dt is _BF16 else 0, k.data_ptr(), kr, kh, v.data_ptr(), vr, vh, qp, qr, qh, yp,
                           n_q * hd, hd, n_q, cp, sp, n_pos, rot, ROPE_LAYOUTS[layout], _raw_stream(dev))
    if rc:
        _check(rc)
    return True, y


def kv8_append(cache, k, v, page_tab, seq_len, seq_off=None, q=None, cos=None, sin=None, layout: str = "half",
               q_out=None, tab_row=None, stream=None):
    """Appends keys and values (bf16 or fp32 [rows, n_kv, head_dim], rows and
    heads at any strides) to their sequences in ``cache``, keys turned by their
    positions with the rope_table (cos, sin) where one is given, and returns q
    turned likewise (into ``q_out``, which may be q but must not overlap k, v or q
    in any other way), or None without q.
      page_tab  int32 [sequences, pages]: each sequence's pages in order
                (``tab_row`` int32 [sequences] picks rows of a larger table)
      seq_len   int32 [sequences]: tokens of each, the new rows counted
      seq_off   int32 [sequences + 1]: each sequence's rows, or None for one
                row a sequence
    Not recorded by autograd: the cache and the result carry no gradient.
    See rg_kv8_append in rollout.h for scales, rounding and what padding gets."""
    lib = _ready or _library()
    if q_out is None and stream is None:
        try:
            done, y = _append_now(lib, cache, k, v, page_tab, seq_len, seq_off, q, cos, sin, layout, tab_row)
        except AttributeError:
            done = False
        if done:
            return y
    dt, code = _float_type("k", k)
    c = _cache_args(cache)
    rows = k.shape[0]
    _view("k", k, dt, (rows, c.n_kv, c.head_dim))
    _view("v", v, dt, (rows, c.n_kv, c.head_dim))
    b = _batch_args(rows, page_tab, seq_len, seq_off, tab_row)
    rot = 0
    if cos is not None or sin is not None:
        rot = _tables(cos, sin, c.head_dim, layout)
    n_q = 0
    if q is not None:
        if _float_type("q", q)[0] != dt:
            raise TypeError(f"q must have dtype {dt}, got {q.dtype}")
        n_q = q.shape[1]
        _sizes(heads=n_q)
        _view("q", q, dt, (rows, n_q, c.head_dim))
        if n_q < 1 or n_q % c.n_kv:
            raise ValueError(f"q must have a multiple of {c.n_kv} heads, got {n_q}")
        if q_out is not None:
            _written("q_out", _view("q_out", q_out, dt, q.shape))
    elif q_out is not None:
        raise ValueError("q_out is given without q")
    _one_device(dict(k=k, v=v, q=q, q_out=q_out, cos=cos, sin=sin, page_tab=page_tab, seq_len=seq_len, seq_off=seq_off,
                     tab_row=tab_row, **{"cache." + n: t for n, t in zip(Kv8Cache._fields, cache)}))
    dev = k.device
    with _On(dev):
        if q is not None and q_out is None:
            q_out = _empty(q, tuple(q.shape), dt, stream)
        qa = (0, 0, 0, 0, 0, 0) if q is None else (q.data_ptr(), q.stride(0), q.stride(1), q_out.data_ptr(),
                                                   q_out.stride(0), q_out.stride(1))
        ta = (0, 0, 0, 0, 0) if rot == 0 else (cos.data_ptr(), sin.data_ptr(), cos.shape[0], rot, ROPE_LAYOUTS[layout])
        _check(lib.rg_kv8_append(C.byref(c), C.byref(b), code, k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(),
                                 v.stride(0), v.stride(1), *qa, n_q, *ta, _stream(dev, stream)))
    return q_out


def _attention_now(lib, cache, q, page_tab, seq_len, seq_off, max_len, scale, tab_row):
    """The call where every argument is in place, else None."""
    dt, dev = q.dtype, q.get_device()
    if not ((dt is _BF16 or dt is _F32) and dev >= 0 and _device() == dev and q.dim() == 3):
        return None
    rows, n_q, hd = q.shape
    qr, qh, q1 = q.stride()
    c = _cache_fits(cache, dev)
    b = _batch_fits(rows, page_tab, seq_len, seq_off, tab_row, dev)
    if c is None or b is None:
        return None
    c, n_kv, head_dim, page = c
    b, n_seqs, stride = b
    bound = max(1, stride * page) if max_len is None else int(max_len)
    if not (hd == head_dim and q1 == 1 and 0 < n_q <= _MOST and n_q % n_kv == 0 and 1 <= bound <= 1 << 30):
        return None
    y = _dense(q, (rows, n_q, hd))
    need = lib.rg_kv8_attention_scratch(n_q, n_kv, hd, rows, n_seqs, 0 if seq_off is None else 1, bound)
    scratch, sp = None, 0
    if need > 0:
        scratch = q.new_empty(need // 4, dtype=_F32)
        sp = scratch.data_ptr()
    rc = lib.rg_kv8_attention(c, b, 1 if dt is _BF16 else 0, q.data_ptr(), qr, qh, n_q, y.data_ptr(),
                              hd ** -0.5 if scale is None else float(scale), bound, sp, need, _raw_stream(dev))
    if rc:
        _check(rc)
    return y


def kv8_attention(cache, q, page_tab, seq_len, seq_off=None, max_len: Optional[int] = None,
                  scale: Optional[float] = None, out=None, tab_row=None, stream=None):
    """Causal attention of q (bf16 or fp32 [rows, n_q, head_dim], rows and heads
    at any strides, turned already) over the sequences' tokens in ``cache``, the
    rows' own included.  Rows and sequences as for kv8_append.  ``max_len``
    bounds seq_len (None: what the page table can hold; a close bound makes
    better launches), ``scale`` defaults to 1/sqrt(head_dim).  Returns
    [rows, n_q, head_dim] in q's dtype, zeros for padding rows; rows past the
    last sequence's are not written.  Not recorded by autograd: the result
    carries no gradient.  See rg_kv8_attention in rollout.h."""
    lib = _ready or _library()
    if out is None and stream is None:
        try:
            y = _attention_now(lib, cache, q, page_tab, seq_len, seq_off, max_len, scale, tab_row)
        except AttributeError:
            y = None
        if y is not None:
            return y
    dt, code = _float_type("q", q)
    c = _cache_args(cache)
    rows, n_q, hd = q.shape
    _sizes(heads=n_q)
    _view("q", q, dt, (rows, n_q, c.head_dim))
    if n_q < 1 or n_q % c.n_kv:
        raise ValueError(f"q must have a multiple of {c.n_kv} heads, got {n_q}")
    b = _batch_args(rows, page_tab, seq_len, seq_off, tab_row)
    max_len = max(1, b.tab_stride * c.page_tokens) if max_len is None else int(max_len)
    if max_len < 1 or max_len > 1 << 30:
        raise ValueError(f"max_len must be in [1, 2^30], got {max_len}")
    if out is not None:
        _dev("out", out, dt, (rows, n_q, hd))
    _one_device(dict(q=q, out=out, page_tab=page_tab, seq_len=seq_len, seq_off=seq_off, tab_row=tab_row,
                     **{"cache." + n: t for n, t in zip(Kv8Cache._fields, cache)}))
    dev = q.device
    with _On(dev):
        if out is None:
            out = _empty(q, (rows, n_q, hd), dt, stream)
        need = lib.rg_kv8_attention_scratch(n_q, c.n_kv, hd, rows, b.n_seqs, 0 if seq_off is None else 1, max_len)
        _check(min(need, 0))
        scratch = _empty(q, (need // 4,), _F32, stream) if need else None
        _check(lib.rg_kv8_attention(C.byref(c), C.byref(b), code, q.data_ptr(), q.stride(0), q.stride(1), n_q,
                                    out.data_ptr(), hd ** -0.5 if scale is None else float(scale), max_len,
                                    0 if scratch is None else scratch.data_ptr(), need, _stream(dev, stream)))
    return out
