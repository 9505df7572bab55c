"""What the calls on drafted trees and the sampler refuse: by the binding's checks
and by the library's own, all before any device work (CPU only; the addresses handed
to the library are stand-ins that nothing reads)."""
import ctypes as C
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2606_02218_amd", "librollout.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="library not built")
I32, I64 = torch.int32, torch.int64


def _args(rows=5, n_q=4, hd=64, n=2):
    import paper_2606_02218_amd as rg
    cache = rg.Kv8Cache.empty(8, 2, hd, 16, device="cpu")
    return dict(cache=cache, q=torch.zeros(rows, n_q, hd, dtype=torch.bfloat16), page_tab=torch.zeros(n, 3, dtype=I32),
                seq_len=torch.ones(n, dtype=I32), seq_off=torch.zeros(n + 1, dtype=I32), mask=torch.zeros(rows, 1, dtype=I64))


def test_tree_refuses():
    import paper_2606_02218_amd as rg
    p, n, off = torch.zeros(5, dtype=I32), torch.ones(2, dtype=I32), torch.zeros(3, dtype=I32)
    with pytest.raises(TypeError, match="GPU memory"):
        rg.kv8_tree(p, n, off)
    with pytest.raises(TypeError, match="parent"):
        rg.kv8_tree(p.long(), n, off)
    with pytest.raises(TypeError, match="torch.Tensor"):
        rg.kv8_tree([0], n, off)
    with pytest.raises(ValueError, match="parent"):
        rg.kv8_tree(p[None], n, off)
    with pytest.raises(ValueError, match="seq_off"):
        rg.kv8_tree(p, n, off[:2])
    with pytest.raises(ValueError, match="contiguous"):
        rg.kv8_tree(torch.zeros(10, dtype=I32)[::2], n, off)
    for words in (0, 65):
        with pytest.raises(ValueError, match="1 to 64 words"):
            rg.kv8_tree(p, n, off, words=words)


@pytest.mark.parametrize("change,error,match", [
    (dict(q=torch.zeros(5, 4, 64, dtype=torch.float16)), TypeError, "dtype"), (dict(q=torch.zeros(5, 3, 64)), ValueError, "multiple of 2"),
    (dict(q=torch.zeros(5, 4, 32)), ValueError, "q must have shape"), (dict(q=torch.zeros(5, 64, 4).transpose(1, 2)), ValueError, "last dim"),
    (dict(seq_off=None), ValueError, "seq_off is required"), (dict(seq_off=torch.zeros(4, dtype=I32)), ValueError, "seq_off"),
    (dict(mask=torch.zeros(5, 1, dtype=I32)), TypeError, "mask"), (dict(mask=torch.zeros(4, 1, dtype=I64)), ValueError, "mask must have a row"),
    (dict(mask=torch.zeros(5, 65, dtype=I64)), ValueError, "1 to 64 words"), (dict(mask=torch.zeros(5, 0, dtype=I64)), ValueError, "1 to 64 words"),
    (dict(mask=torch.zeros(5, dtype=I64)), ValueError, "mask"), (dict(mask=torch.zeros(5, 4, dtype=I64)[:, ::2]), ValueError, "contiguous"),
    (dict(max_len=0), ValueError, "max_len"), (dict(max_len=(1 << 30) + 1), ValueError, "max_len"),
    (dict(out=torch.zeros(5, 4, 64)), TypeError, "out"), (dict(out=torch.zeros(4, 4, 64, dtype=torch.bfloat16)), ValueError, "out"),
    (dict(tab_row=torch.zeros(3, dtype=I32)), ValueError, "tab_row"), (dict(page_tab=torch.zeros(1, 3, dtype=I32)), ValueError, "page_tab"),
    (dict(), TypeError, "GPU memory")])
def test_attention_refuses(change, error, match):
    import paper_2606_02218_amd as rg
    with pytest.raises(error, match=match):
        rg.kv8_tree_attention(**{**_args(), **change})


@pytest.mark.parametrize("change,error,match", [
    (dict(last=torch.zeros(2, dtype=I64)), TypeError, "last"), (dict(last=torch.zeros(3, dtype=I32)), ValueError, "last"),
    (dict(seq_off=None), ValueError, "seq_off is required"), (dict(mask=torch.zeros(5, 65, dtype=I64)), ValueError, "words"),
    (dict(mask=torch.zeros(5, 1)), TypeError, "mask"), (dict(page_tab=torch.zeros(1, 3, dtype=I32)), ValueError, "page_tab"),
    (dict(), TypeError, "GPU memory")])
def test_accept_refuses(change, error, match):
    import paper_2606_02218_amd as rg
    a = {**_args(), "last": torch.zeros(2, dtype=I32), **change}
    del a["q"]
    with pytest.raises(error, match=match):
        rg.kv8_accept(**a)


@pytest.mark.parametrize("change,error,match", [
    (dict(logits=torch.zeros(3, 9).half()), TypeError, "logits must have dtype"), (dict(logits=[1]), TypeError, "torch.Tensor"),
    (dict(logits=torch.zeros(9)), ValueError, "2 dimensions"), (dict(logits=torch.zeros(9, 3).T), ValueError, "last dimension"),
    (dict(logits=torch.zeros(3, 0)), ValueError, "vocab"), (dict(logits=torch.zeros(1, 1).expand(3, (1 << 20) + 1).contiguous()), ValueError, "vocab"),
    (dict(u=torch.zeros(3).half()), TypeError, "u must have dtype"), (dict(u=torch.zeros(4)), ValueError, "u must have shape"),
    (dict(u=torch.zeros(6)[::2]), ValueError, "contiguous"), (dict(temperature=-0.1), ValueError, "temperature"),
    (dict(temperature=float("inf")), ValueError, "temperature"), (dict(temperature=float("nan")), ValueError, "temperature"),
    (dict(top_k=-1), ValueError, "top_k"), (dict(top_k=2 ** 63), ValueError, "top_k"), (dict(top_p=0.0), ValueError, "top_p"),
    (dict(top_p=1.1), ValueError, "top_p"), (dict(min_p=-0.1), ValueError, "min_p"), (dict(min_p=1.5), ValueError, "min_p"),
    (dict(min_p=float("nan")), ValueError, "min_p"), (dict(temperature=torch.ones(4)), ValueError, "temperature"),
    (dict(top_k=torch.ones(3)), TypeError, "top_k"), (dict(top_p=torch.ones(3).double()), TypeError, "top_p"),
    (dict(min_p=torch.ones(6)[::2]), ValueError, "min_p"), (dict(), TypeError, "GPU memory"),
    (dict(temperature=torch.ones(3)), TypeError, "GPU memory")])
def test_sample_refuses(change, error, match):
    import paper_2606_02218_amd as rg
    with pytest.raises(error, match=match):
        rg.sample(**{**dict(logits=torch.zeros(3, 9), u=torch.zeros(3)), **change})


def test_sizes_past_the_librarys_integers():
    import paper_2606_02218_amd as rg
    many, one = 2 ** 31 + 3, torch.zeros(1, dtype=I32)
    with pytest.raises(ValueError, match="below 2\\^31"):
        rg.sample(torch.zeros(1, 9).expand(many, 9), torch.zeros(1))
    a = _args(1, n=1)
    with pytest.raises(ValueError, match="below 2\\^31"):
        rg.kv8_tree_attention(**{**a, "q": a["q"].expand(1, 4, 64)[:, :1].expand(1, 2 * many, 64)})
    with pytest.raises(ValueError, match="below 2\\^31"):
        rg.kv8_tree_attention(**{**a, "q": a["q"].expand(many, 4, 64), "mask": torch.zeros(1, 1, dtype=I64).expand(many, 1)})


# ---------------------------------------------------------------- the library's own checks
def _lib():
    from paper_2606_02218_amd import _draft
    return _draft._library()


def _cache(**change):
    from paper_2606_02218_amd import _kv8
    f = dict(k=1 << 12, v=1 << 13, k_scale=1 << 14, v_scale=1 << 15, pages=8, n_kv=2, head_dim=64, page_tokens=16)
    return _kv8.rg_kv8_cache(*{**f, **change}.values())


def _batch(**change):
    from paper_2606_02218_amd import _kv8
    f = dict(page_tab=1 << 16, tab_rows=2, tab_stride=3, tab_row=0, seq_off=1 << 17, seq_len=1 << 18, n_seqs=2, rows=5)
    return _kv8.rg_kv8_batch(*{**f, **change}.values())


def _refused(rc, code, text):
    lib = _lib()
    assert rc == code and text in lib.rg_last_error(), (rc, lib.rg_last_error())


def test_library_refuses_trees():
    lib = _lib()
    p = [C.c_void_p(1 << (20 + i)) for i in range(8)]
    tree = lambda **c: lib.rg_kv8_tree(*{**dict(a=p[0], b=p[1], c=p[2], n=2, rows=5, words=1, m=p[3], pos=p[4], st=None), **c}.values())  # noqa: E731
    for c, text in [(dict(words=0), b"words"), (dict(words=65), b"words"), (dict(rows=-1), b"rows"), (dict(n=-1), b"rows or n_seqs"),
                    (dict(n=(1 << 24) + 1), b"n_seqs"), (dict(a=None), b"NULL"), (dict(m=None), b"NULL"), (dict(pos=None), b"NULL"),
                    (dict(b=None), b"NULL"), (dict(c=None), b"NULL")]:
        _refused(tree(**c), -1, text)
    assert tree(rows=0) == 0 and tree(n=0) == 0 and tree(rows=0, a=None, m=None) == 0


def test_library_refuses_attention():
    lib = _lib()
    p = [C.c_void_p(1 << (20 + i)) for i in range(8)]

    def call(cache=None, batch=None, **c):
        f = dict(dtype=1, q=p[0], qr=256, qh=64, n_q=4, mask=p[1], words=1, out=p[2], scale=0.1, max_len=40, scratch=None, need=0, st=None)
        return lib.rg_kv8_tree_attention(C.byref(_cache(**(cache or {}))), C.byref(_batch(**(batch or {}))), *{**f, **c}.values())
    for c, code, text in [
            (dict(dtype=2), -1, b"dtype"), (dict(n_q=3), -1, b"multiple"), (dict(n_q=0), -1, b"multiple"), (dict(n_q=258), -4, b"128"),
            (dict(scale=0.0), -1, b"scale"), (dict(scale=3e38), -1, b"scale"), (dict(scale=float("nan")), -1, b"scale"),
            (dict(max_len=0), -1, b"max_len"), (dict(words=0), -1, b"words"), (dict(words=65), -1, b"words"), (dict(q=None), -1, b"NULL"),
            (dict(mask=None), -1, b"NULL"), (dict(out=None), -1, b"NULL"), (dict(out=C.c_void_p(1 << 20 | 8)), -1, b"aligned"),
            (dict(max_len=1 << 20), -1, b"scratch"), (dict(max_len=1 << 20, scratch=p[4], need=64), -1, b"scratch"),
            (dict(batch=dict(seq_off=0)), -1, b"seq_off"), (dict(batch=dict(tab_stride=1 << 28)), -1, b"2^30"),
            (dict(batch=dict(n_seqs=0)), -1, b"n_seqs"), (dict(batch=dict(page_tab=0)), -1, b"NULL"),
            (dict(cache=dict(head_dim=96)), -4, b"head_dim"), (dict(cache=dict(page_tokens=24)), -4, b"page_tokens"),
            (dict(cache=dict(k=0)), -1, b"NULL"), (dict(cache=dict(v=8)), -1, b"aligned")]:
        _refused(call(**c), code, text)
    assert call(batch=dict(rows=0)) == 0
    s = lib.rg_kv8_tree_attention_scratch
    assert s(1, 12, 2, 128, 0, 0, 1, 100) == 0 and s(1, 12, 2, 128, 30, 1, 1, 100000) > 0
    for a in [(3, 12, 2, 128, 4, 1, 1, 9), (1, 12, 5, 128, 4, 1, 1, 9), (1, 12, 2, 128, -1, 1, 1, 9), (1, 12, 2, 128, 4, 1, 1, 0),
              (1, 0, 1, 64, 1, 1, 1, 1), (1, 12, 2, 128, 4, 1, 0, 9), (1, 12, 2, 128, 4, 1, 65, 9), (1, 129, 1, 64, 1, 1, 1, 9)]:
        assert s(*a) == -1


def test_bounds_past_a_tables_most_ask_for_no_chunk_more():
    s = _lib().rg_kv8_tree_attention_scratch
    for a in [(1, 12, 2, 128, 100000, 10, 1), (0, 12, 2, 128, 100000, 10, 1), (1, 28, 4, 128, 128, 2, 1), (1, 2, 1, 64, 3, 1, 1)]:
        assert s(*a, 2 ** 31 - 1) == s(*a, 1 << 30)
    assert s(1, 12, 2, 128, 100000, 10, 1, 2 ** 31 - 1) == 0


def test_library_refuses_accept():
    lib = _lib()
    p = [C.c_void_p(1 << (20 + i)) for i in range(8)]

    def call(cache=None, batch=None, **c):
        f = dict(mask=p[1], words=1, last=p[2], new=p[3], st=None)
        return lib.rg_kv8_accept(C.byref(_cache(**(cache or {}))), C.byref(_batch(**(batch or {}))), *{**f, **c}.values())
    for c, text in [(dict(words=0), b"words"), (dict(mask=None), b"NULL"), (dict(last=None), b"NULL"), (dict(new=None), b"NULL"),
                    (dict(batch=dict(seq_off=0)), b"seq_off"), (dict(new=C.c_void_p(1 << 18)), b"overlaps"),
                    (dict(new=C.c_void_p((1 << 18) - 4)), b"overlaps"), (dict(new=p[2]), b"overlaps"),
                    (dict(new=C.c_void_p((1 << 16) + 20)), b"overlaps"), (dict(new=C.c_void_p((1 << 17) + 8)), b"overlaps"),
                    (dict(batch=dict(seq_len=0, rows=0)), b"NULL")]:
        _refused(call(**c), -1, text)
    assert call(batch=dict(n_seqs=0, rows=0)) == 0


def test_library_refuses_lengths_in_masks_and_caches():
    """new_len on what the accept reads beyond the batch: the first and the last four bytes of each, and next to them."""
    lib = _lib()
    at = lambda i: 1 << (30 + i)  # noqa: E731
    cache = _cache(k=at(1), v=at(2), k_scale=at(3), v_scale=at(4))           # 16 blocks of 1024 codes
    call = lambda new: lib.rg_kv8_accept(C.byref(cache), C.byref(_batch()), at(0), 3, at(5), new, None)  # noqa: E731
    for i, size in ((0, 5 * 3 * 8), (1, 16 << 10), (2, 16 << 10), (3, 64), (4, 64), (5, 8)):
        for new in (at(i) - 4, at(i), at(i) + size - 4):
            _refused(call(new), -1, b"overlaps")


def test_library_refuses_samples():
    from paper_2606_02218_amd import _draft
    lib = _lib()
    p = [C.c_void_p(1 << (20 + i)) for i in range(8)]

    def call(options=True, t=1.0, k=0, tp=1.0, mp=0.0, **c):
        o = _draft.rg_sample_options(t, tp, mp, k, None, None, None, None)
        f = dict(dtype=1, z=p[0], step=100, rows=3, vocab=100, ut=0, u=p[1], o=C.byref(o) if options else None, tok=p[2], lp=p[3],
                 kp=p[4], scratch=p[5], need=1 << 20, st=None)
        return lib.rg_sample(*{**f, **c}.values())
    for c, code, text in [
            (dict(options=False), -1, b"NULL"), (dict(dtype=2), -1, b"dtype"), (dict(ut=1), -1, b"fp32 or fp64"), (dict(rows=-1), -1, b"rows"),
            (dict(vocab=0), -1, b"vocab"), (dict(vocab=(1 << 20) + 1), -4, b"2^20"), (dict(t=-1.0), -1, b"temperature"),
            (dict(t=float("inf")), -1, b"temperature"), (dict(t=float("nan")), -1, b"temperature"), (dict(k=-1), -1, b"top_k"),
            (dict(tp=0.0), -1, b"top_p"), (dict(tp=1.5), -1, b"top_p"), (dict(tp=float("nan")), -1, b"top_p"), (dict(mp=-0.5), -1, b"min_p"),
            (dict(mp=1.5), -1, b"min_p"), (dict(z=None), -1, b"NULL"), (dict(u=None), -1, b"NULL"), (dict(tok=None), -1, b"NULL"),
            (dict(lp=None), -1, b"NULL"), (dict(kp=None), -1, b"NULL"), (dict(scratch=None), -1, b"scratch"),
            (dict(need=8), -1, b"scratch"), (dict(scratch=C.c_void_p(1 << 20 | 4)), -1, b"aligned")]:
        _refused(call(**c), code, text)
    assert call(rows=0, z=None) == 0
    plain, cut = _draft.rg_sample_options(1.0, 1.0, 0.0, 0), _draft.rg_sample_options(1.0, 0.9, 0.0, 0)
    size = lambda rows, vocab, o=plain: lib.rg_sample_scratch(rows, vocab, C.byref(o))  # noqa: E731
    assert size(0, 5) == 0 and 0 < size(4, 1 << 20) < size(4, 1 << 20, cut)
    for a in [(-1, 5), (1, 0), (1, (1 << 20) + 1)]:
        assert size(*a) == -1
    assert lib.rg_sample_scratch(1, 5, None) == -1
