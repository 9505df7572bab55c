"""ctypes marshalling for drafted trees over the 8-bit key/value cache and for
sampling from given logits (include/rollout.h).  No computation happens here."""
from __future__ import annotations

import ctypes as C
import struct
from typing import Optional

from . import _kv8
from ._kv8 import (Kv8Cache, _batch_args, _batch_fits, _cache_args, _cache_fits, _dense, _empty, _float_type, _MOST, _On, _one_device,
                   _sizes, _stream, _view)
from ._lib import _check, _dev


class rg_sample_options(C.Structure):
    _fields_ = [("temperature", C.c_double), ("top_p", C.c_double), ("min_p", C.c_double), ("top_k", C.c_int64),
                ("temperature_rows", C.c_void_p), ("top_k_rows", C.c_void_p), ("top_p_rows", C.c_void_p),
                ("min_p_rows", C.c_void_p)]


_OPTIONS = struct.Struct("@3dq4P").pack
_P, _I, _L = C.c_void_p, C.c_int32, C.c_int64
_ARGS = {
    "rg_kv8_tree": ([_P, _P, _P, _I, _I, _I, _P, _P, _P], C.c_int),
    "rg_kv8_tree_attention_scratch": ([_I] * 8, _L),
    "rg_kv8_tree_attention": ([_P, _P, _I, _P, _L, _L, _I, _P, _I, _P, C.c_float, _I, _P, _L, _P], C.c_int),
    "rg_kv8_accept": ([_P, _P, _P, _I, _P, _P, _P], C.c_int),
    "rg_sample_scratch": ([_I, _I, _P], _L),
    "rg_sample": ([_I, _P, _L, _I, _I, _I, _P, _P, _P, _P, _P, _P, _L, _P], C.c_int),
}
WORDS = 64              # most words of a row's mask
_MOST_VOCAB = 1 << 20
_ready = None
_BF16 = _F32 = _F64 = _I32 = _I64 = _device = _raw_stream = _make = None


def _library():
    global _ready, _BF16, _F32, _F64, _I32, _I64, _device, _raw_stream, _make
    if _ready is None:
        lib = _kv8._library()
        for name, (args, res) in _ARGS.items():
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = args, res
        import torch
        _BF16, _F32, _F64, _I32, _I64 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64
        _device, _raw_stream, _make = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream, torch.empty
        _ready = lib
    return _ready


# As for the cache's other calls: each asks in few questions whether every argument is
# in place, and only where that fails goes through the checks that say what is wrong.
def _mask_fits(mask, rows, dev):
    """Words of a mask that is in place, or None."""
    if not (mask.dtype is _I64 and mask.get_device() == dev and mask.is_contiguous()):
        return None
    n, words = mask.shape
    return words if n == rows and 1 <= words <= WORDS else None


def _mask_args(mask, rows):
    _dev("mask", mask, _I64, ndim=2)
    if mask.shape[0] != rows:
        raise ValueError(f"mask must have a row for each of {rows} nodes, got shape {tuple(mask.shape)}")
    words = int(mask.shape[1])
    if not 1 <= words <= WORDS:
        raise ValueError(f"a mask has 1 to {WORDS} words a row, got {words}")
    return words


def _tree_now(lib, parent, seq_len, seq_off, words):
    dev = parent.get_device()
    if not (parent.dtype is seq_len.dtype is seq_off.dtype is _I32 and dev >= 0 and _device() == dev and
            seq_len.get_device() == seq_off.get_device() == dev and parent.is_contiguous() and seq_len.is_contiguous() and
            seq_off.is_contiguous()):
        return None
    (rows,), (n,), (n1,) = parent.shape, seq_len.shape, seq_off.shape
    if not (n1 == n + 1 and rows <= _MOST and 1 <= words <= WORDS):
        return None
    mask = parent.new_empty((rows, words), dtype=_I64)
    pos = parent.new_empty((rows,))
    rc = lib.rg_kv8_tree(parent.data_ptr(), seq_off.data_ptr(), seq_len.data_ptr(), n, rows, words, mask.data_ptr(),
                         pos.data_ptr(), _raw_stream(dev))
    if rc:
        _check(rc)
    return mask, pos


def kv8_tree(parent, seq_len, seq_off, words: int = 1, stream=None):
    """What each drafted token sees of its tree, and where it stands: (mask, pos).
      parent   int32 [rows]: each node's parent, by its number among its
               sequence's nodes; -1 behind the context
      seq_len  int32 [sequences]: tokens of each, the nodes counted
      seq_off  int32 [sequences + 1]: each sequence's nodes
    ``mask`` is int64 [rows, words], bit i % 64 of word i / 64 for node i: its
    own and its ancestors'.  A word holds 64 nodes and those past the last word have no
    bit, so that no node sees them, not even they themselves: a tree of more than 64
    nodes needs ``words`` of nodes / 64, rounded up.  ``pos`` is int32 [rows], the
    context's length plus the node's depth.  Rows past the last sequence's are not
    written.  See rg_kv8_tree in rollout.h for padding and for parents that are none."""
    lib = _ready or _library()
    if stream is None:
        try:
            got = _tree_now(lib, parent, seq_len, seq_off, words)
        except (AttributeError, TypeError, ValueError):
            got = None
        if got is not None:
            return got
    _dev("parent", parent, _I32, ndim=1)
    _dev("seq_len", seq_len, _I32, ndim=1)
    rows, n, words = parent.shape[0], seq_len.shape[0], int(words)
    _dev("seq_off", seq_off, _I32, (n + 1,))
    _sizes(rows=rows, sequences=n)
    if not 1 <= words <= WORDS:
        raise ValueError(f"a mask has 1 to {WORDS} words a row, got {words}")
    _one_device(dict(parent=parent, seq_len=seq_len, seq_off=seq_off))
    with _On(parent.device):
        mask, pos = _empty(parent, (rows, words), _I64, stream), _empty(parent, (rows,), _I32, stream)
        _check(lib.rg_kv8_tree(parent.data_ptr(), seq_off.data_ptr(), seq_len.data_ptr(), n, rows, words, mask.data_ptr(),
                               pos.data_ptr(), _stream(parent.device, stream)))
    return mask, pos


def _attention_now(lib, cache, q, page_tab, seq_len, seq_off, mask, max_len, scale, tab_row):
    dt, dev = q.dtype, q.get_device()
    if not ((dt is _BF16 or dt is _F32) and dev >= 0 and _device() == dev and q.dim() == 3 and seq_off is not None):
        return None
    rows, n_q, hd = q.shape
    qr, qh, q1 = q.stride()
    c = _cache_fits(cache, dev)
    b = _batch_fits(rows, page_tab, seq_len, seq_off, tab_row, dev)
    words = _mask_fits(mask, rows, dev)
    if c is None or b is None or words is None:
        return None
    c, n_kv, head_dim, page = c
    b, n_seqs, stride = b
    bound = max(1, stride * page) if max_len is None else int(max_len)
    if not (hd == head_dim and q1 == 1 and 0 < n_q <= _MOST and n_q % n_kv == 0 and 1 <= bound <= 1 << 30):
        return None
    y = _dense(q, (rows, n_q, hd))
    code = 1 if dt is _BF16 else 0
    need = lib.rg_kv8_tree_attention_scratch(code, n_q, n_kv, hd, rows, n_seqs, words, bound)
    scratch, sp = None, 0
    if need > 0:
        scratch = q.new_empty(need // 4, dtype=_F32)
        sp = scratch.data_ptr()
    rc = lib.rg_kv8_tree_attention(c, b, code, q.data_ptr(), qr, qh, n_q, mask.data_ptr(), words, y.data_ptr(),
                                   hd ** -0.5 if scale is None else float(scale), bound, sp, need, _raw_stream(dev))
    if rc:
        _check(rc)
    return y


def kv8_tree_attention(cache, q, page_tab, seq_len, seq_off, mask, max_len: Optional[int] = None,
                       scale: Optional[float] = None, out=None, tab_row=None, stream=None):
    """Attention of drafted tokens q (bf16 or fp32 [rows, n_q, head_dim], rows
    and heads at any strides, turned already) over their sequences' contexts in
    ``cache`` and the nodes that ``mask`` (int64 [rows, words], as kv8_tree gives it)
    shows them.  Rows, sequences and the rest as for kv8_attention; the rows'
    keys and values are in the cache already, node i in slot seq_len - n + i.
    Returns [rows, n_q, head_dim] in q's dtype, zeros for rows that see nothing;
    rows past the last sequence's are not written.  Not recorded by autograd: the
    result carries no gradient.  See rg_kv8_tree_attention in rollout.h."""
    lib = _ready or _library()
    if out is None and stream is None:
        try:
            y = _attention_now(lib, cache, q, page_tab, seq_len, seq_off, mask, max_len, scale, tab_row)
        except (AttributeError, ValueError):
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
    if seq_off is None:
        raise ValueError("seq_off is required: it says which nodes are a sequence's")
    b = _batch_args(rows, page_tab, seq_len, seq_off, tab_row)
    words = _mask_args(mask, rows)
    max_len = max(1, b.tab_stride * c.page_tokens) if max_len is None else int(max_len)
    if max_len < 1 or max_len > 1 << 30:
        raise ValueError(f"max_len must be in [1, 2^30], got {max_len}")
    if out is not None:
        _dev("out", out, dt, (rows, n_q, hd))
    _one_device(dict(q=q, out=out, page_tab=page_tab, seq_len=seq_len, seq_off=seq_off, tab_row=tab_row, mask=mask,
                     **{"cache." + n: t for n, t in zip(Kv8Cache._fields, cache)}))
    dev = q.device
    with _On(dev):
        if out is None:
            out = _empty(q, (rows, n_q, hd), dt, stream)
        need = lib.rg_kv8_tree_attention_scratch(code, n_q, c.n_kv, hd, rows, b.n_seqs, words, max_len)
        _check(min(need, 0))
        scratch = _empty(q, (need // 4,), _F32, stream) if need else None
        _check(lib.rg_kv8_tree_attention(C.byref(c), C.byref(b), code, q.data_ptr(), q.stride(0), q.stride(1), n_q,
                                         mask.data_ptr(), words, out.data_ptr(), hd ** -0.5 if scale is None else float(scale),
                                         max_len, 0 if scratch is None else scratch.data_ptr(), need, _stream(dev, stream)))
    return out


def _accept_now(lib, cache, page_tab, seq_len, seq_off, mask, last, tab_row):
    dev = seq_len.get_device()
    if not (dev >= 0 and _device() == dev and seq_off is not None and last.dtype is _I32 and last.get_device() == dev and
            last.is_contiguous() and last.shape == seq_len.shape):
        return None
    rows = mask.shape[0]
    c = _cache_fits(cache, dev)
    b = _batch_fits(rows, page_tab, seq_len, seq_off, tab_row, dev)
    words = _mask_fits(mask, rows, dev)
    if c is None or b is None or words is None:
        return None
    new = seq_len.new_empty(seq_len.shape)
    rc = lib.rg_kv8_accept(c[0], b[0], mask.data_ptr(), words, last.data_ptr(), new.data_ptr(), _raw_stream(dev))
    if rc:
        _check(rc)
    return new


def kv8_accept(cache, page_tab, seq_len, seq_off, mask, last, tab_row=None, stream=None):
    """Takes over accepted nodes: those that the mask of each sequence's node
    ``last`` (int32 [sequences], its number among the sequence's nodes, -1: none)
    has a bit for move, in their order, to the slots behind the context in ``cache``.
    The rest as for kv8_tree_attention.  Returns int32 [sequences], the tokens
    that each holds then.  See rg_kv8_accept in rollout.h for scales and rounding."""
    lib = _ready or _library()
    if stream is None:
        try:
            new = _accept_now(lib, cache, page_tab, seq_len, seq_off, mask, last, tab_row)
        except (AttributeError, ValueError):
            new = None
        if new is not None:
            return new
    c = _cache_args(cache)
    _dev("mask", mask, _I64, ndim=2)
    rows = mask.shape[0]
    if seq_off is None:
        raise ValueError("seq_off is required: it says which nodes are a sequence's")
    b = _batch_args(rows, page_tab, seq_len, seq_off, tab_row)
    words = _mask_args(mask, rows)
    _dev("last", last, _I32, (b.n_seqs,))
    _one_device(dict(page_tab=page_tab, seq_len=seq_len, seq_off=seq_off, tab_row=tab_row, mask=mask, last=last,
                     **{"cache." + n: t for n, t in zip(Kv8Cache._fields, cache)}))
    with _On(seq_len.device):
        new = _empty(seq_len, (b.n_seqs,), _I32, stream)
        _check(lib.rg_kv8_accept(C.byref(c), C.byref(b), mask.data_ptr(), words, last.data_ptr(), new.data_ptr(),
                                 _stream(seq_len.device, stream)))
    return new


def _row_option(x, dtype, rows, dev):
    """The address of a row-by-row setting that is in place; 0 for a number."""
    if x.__class__ is float or x.__class__ is int:
        return 0
    if not (x.dtype is dtype and x.get_device() == dev and x.is_contiguous() and x.shape == (rows,)):
        raise AttributeError
    return x.data_ptr()


def _sample_now(lib, z, u, temperature, top_k, top_p, min_p):
    dt, dev = z.dtype, z.get_device()
    if not ((dt is _BF16 or dt is _F32) and dev >= 0 and _device() == dev):
        return None
    rows, vocab = z.shape
    step, one = z.stride()
    ut = u.dtype
    if not (one == 1 and rows <= _MOST and 1 <= vocab <= _MOST_VOCAB and (ut is _F32 or ut is _F64) and u.get_device() == dev and
            u.is_contiguous() and u.shape == (rows,)):
        return None
    t, k, p, m = (_row_option(temperature, _F32, rows, dev), _row_option(top_k, _I32, rows, dev),
                  _row_option(top_p, _F32, rows, dev), _row_option(min_p, _F32, rows, dev))
    o = _OPTIONS(0.0 if t else temperature, 0.0 if p else top_p, 0.0 if m else min_p, 0 if k else top_k, t, k, p, m)
    need = lib.rg_sample_scratch(rows, vocab, o)
    tokens = u.new_empty((rows,), dtype=_I32)
    lp = u.new_empty((2, rows), dtype=_F32)
    scratch = u.new_empty(need // 4, dtype=_F32)
    at = lp.data_ptr()
    rc = lib.rg_sample(1 if dt is _BF16 else 0, z.data_ptr(), step, rows, vocab, 2 if ut is _F64 else 0, u.data_ptr(), o,
                       tokens.data_ptr(), at, at + 4 * rows, scratch.data_ptr(), need, _raw_stream(dev))
    if rc:
        _check(rc)
    return tokens, lp[0], lp[1]


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, stream=None):
    """Draws a token for every row of ``logits`` (bf16 or fp32 [rows, vocab],
    rows at any stride) with the uniform numbers ``u`` (fp32 or fp64 [rows] in
    [0, 1)): temperature, then what top-k, top-p and min-p leave, then the first
    token, by id, at which the running sum of the kept weights passes u of their sum.
    Each setting is a number or a device tensor with one for every row (fp32
    [rows]; int32 for ``top_k``); top_k 0, top_p 1 and min_p 0 cut nothing,
    temperature 0 takes the largest logit.  Returns (tokens int32 [rows], their
    log-probabilities under softmax(logits / temperature) and under the distribution
    that is left, fp32 [rows] each).  Not recorded by autograd.  See rg_sample in
    rollout.h for ties, NaN and infinities."""
    lib = _ready or _library()
    if stream is None:
        try:
            got = _sample_now(lib, logits, u, temperature, top_k, top_p, min_p)
        except (AttributeError, TypeError, ValueError, struct.error):
            got = None
        if got is not None:
            return got
    import torch
    if not isinstance(logits, torch.Tensor):
        raise TypeError(f"logits must be a torch.Tensor, got {type(logits).__name__}")
    if logits.dtype not in (_BF16, _F32):
        raise TypeError(f"logits must have dtype torch.bfloat16 or torch.float32, got {logits.dtype}")
    if logits.dim() != 2:
        raise ValueError(f"logits must have 2 dimensions [rows, vocab], got shape {tuple(logits.shape)}")
    rows, vocab = logits.shape
    if logits.stride(1) != 1 and vocab != 1:
        raise ValueError("logits must have its last dimension contiguous")
    _sizes(rows=rows)
    if not 1 <= vocab <= _MOST_VOCAB:
        raise ValueError(f"vocab must be in [1, 2^20], got {vocab}")
    _dev("u", u, (_F32, _F64), (rows,))
    tensors = dict(logits=logits, u=u)
    o = rg_sample_options()
    for name, x, dt, lo, hi in (("temperature", temperature, _F32, 0.0, 1.7e308), ("top_k", top_k, _I32, 0, 2 ** 63 - 1),
                                ("top_p", top_p, _F32, 0.0, 1.0), ("min_p", min_p, _F32, 0.0, 1.0)):
        if isinstance(x, torch.Tensor):
            tensors[name] = _dev(name, x, dt, (rows,))
            setattr(o, name + "_rows", x.data_ptr())
            continue
        x = int(x) if dt is _I32 else float(x)
        if not (lo <= x <= hi and (name != "top_p" or x > 0.0)):
            raise ValueError(f"{name} must be in {'(' if name == 'top_p' else '['}{lo}, {hi}], got {x}")
        setattr(o, name, x)
    _one_device(tensors)
    with _On(logits.device):
        need = lib.rg_sample_scratch(rows, vocab, C.byref(o))
        tokens, lp = _empty(u, (rows,), _I32, stream), _empty(u, (2, rows), _F32, stream)
        scratch = _empty(u, (need // 4,), _F32, stream)
        _check(lib.rg_sample(1 if logits.dtype == _BF16 else 0, logits.data_ptr(), logits.stride(0), rows, vocab,
                             2 if u.dtype == _F64 else 0, u.data_ptr(), C.byref(o), tokens.data_ptr(), lp[0].data_ptr(),
                             lp[1].data_ptr(), scratch.data_ptr(), need, _stream(logits.device, stream)))
    return tokens, lp[0], lp[1]
