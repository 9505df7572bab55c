"""What the rotary and 8-bit cache calls refuse: by the binding's checks and by
the library's own, all before any device work (CPU only; the addresses handed
to the library are stand-ins that nothing reads)."""
import ctypes as C
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2606_02218_amd", "librollout.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="library not built")

I32 = torch.int32


def _cache(pages=4, n_kv=2, hd=64, page=16):
    import paper_2606_02218_amd as rg
    return rg.Kv8Cache.empty(pages, n_kv, hd, page, device="cpu")


def _zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def test_rope_refuses():
    import paper_2606_02218_amd as rg
    x, pos, cos = _zeros(3, 2, 64), torch.zeros(3, dtype=I32), torch.zeros(8, 32)
    with pytest.raises(TypeError, match="GPU memory"):
        rg.rope(x, pos, cos, cos)
    with pytest.raises(TypeError, match="dtype"):
        rg.rope(x.half(), pos, cos, cos)
    with pytest.raises(TypeError, match="torch.Tensor"):
        rg.rope([1], pos, cos, cos)
    with pytest.raises(ValueError, match="3 dimensions"):
        rg.rope(x[0], pos, cos, cos)
    with pytest.raises(TypeError, match="pos"):
        rg.rope(x, pos.long(), cos, cos)
    with pytest.raises(ValueError, match="pos"):
        rg.rope(x, pos[:2], cos, cos)
    with pytest.raises(ValueError, match="sin"):
        rg.rope(x, pos, cos, cos[:, :31])
    with pytest.raises(ValueError, match="does not fit"):
        rg.rope(x, pos, torch.zeros(8, 33), torch.zeros(8, 33))
    with pytest.raises(ValueError, match="layout"):
        rg.rope(x, pos, cos, cos, layout="other")
    with pytest.raises(ValueError, match="last dimension"):
        rg.rope(_zeros(3, 64, 2).transpose(1, 2), pos, cos, cos)
    with pytest.raises(ValueError, match="out must have shape"):
        rg.rope(x, pos, cos, cos, out=_zeros(3, 2, 32))
    with pytest.raises(ValueError, match="overlapping"):
        rg.rope(x, pos, cos, cos, out=_zeros(1, 2, 64).expand(3, 2, 64))
    with pytest.raises(ValueError, match="even"):
        rg.rope(_zeros(3, 2, 63), pos, cos[:, :8], cos[:, :8])
    with pytest.raises(ValueError, match="scaling"):
        rg.rope_table(8, 64, scaling="other")
    with pytest.raises(ValueError, match="even rot_dim"):
        rg.rope_table(8, 63)
    with pytest.raises(TypeError, match="GPU memory"):
        rg.rope_table(8, 64, device="cpu")


def test_sizes_past_the_librarys_integers():
    """A size of 2^31 is refused, not wrapped (views without storage: nothing of that size is allocated)."""
    import paper_2606_02218_amd as rg
    many, one, cos = 2 ** 31 + 3, torch.zeros(1, dtype=I32), torch.zeros(8, 32)
    for x in (_zeros(1, 1, 64).expand(many, 1, 64), _zeros(1, 1, 64).expand(1, many, 64)):
        with pytest.raises(ValueError, match="below 2\\^31"):
            rg.rope(x, one, cos, cos)
    with pytest.raises(ValueError, match="below 2\\^31"):
        rg.rope_table(many, 64)
    cache = rg.Kv8Cache.empty(4, 2, 64, device="cpu")
    tab = torch.zeros(1, 1, dtype=I32)
    kv = _zeros(1, 2, 64).expand(many, 2, 64)
    with pytest.raises(ValueError, match="below 2\\^31"):
        rg.kv8_append(cache, kv, kv, tab, one)
    with pytest.raises(ValueError, match="below 2\\^31"):
        rg.kv8_attention(cache, kv, tab, one)
    with pytest.raises(ValueError, match="below 2\\^31"):
        rg.kv8_attention(cache, _zeros(1, 1, 64).expand(1, 2 * many, 64), tab, one)


def test_append_refuses():
    import paper_2606_02218_amd as rg
    c, k = _cache(), _zeros(3, 2, 64)
    tab, n = torch.zeros((3, 2), dtype=I32), torch.ones(3, dtype=I32)
    q = _zeros(3, 4, 64)
    with pytest.raises(TypeError, match="GPU memory"):
        rg.kv8_append(c, k, k, tab, n)
    with pytest.raises(TypeError, match="v must have dtype"):
        rg.kv8_append(c, k, k.float(), tab, n)
    with pytest.raises(ValueError, match="k must have shape"):
        rg.kv8_append(c, _zeros(3, 3, 64), _zeros(3, 3, 64), tab, n)
    with pytest.raises(ValueError, match="one row a sequence"):
        rg.kv8_append(c, k, k, tab, n[:2])
    with pytest.raises(ValueError, match="seq_off"):
        rg.kv8_append(c, k, k, tab, n, torch.zeros(3, dtype=I32))
    with pytest.raises(ValueError, match="a row for each"):
        rg.kv8_append(c, k, k, tab[:2], n)
    with pytest.raises(ValueError, match="tab_row"):
        rg.kv8_append(c, k, k, tab, n, tab_row=n[:1])
    with pytest.raises(TypeError, match="q must have dtype"):
        rg.kv8_append(c, k, k, tab, n, q=q.float())
    with pytest.raises(ValueError, match="multiple of 2 heads"):
        rg.kv8_append(c, k, k, tab, n, q=_zeros(3, 3, 64))
    with pytest.raises(ValueError, match="without q"):
        rg.kv8_append(c, k, k, tab, n, q_out=q)
    with pytest.raises(ValueError, match="q_out must have shape"):
        rg.kv8_append(c, k, k, tab, n, q=q, q_out=_zeros(3, 2, 64))
    with pytest.raises(ValueError, match="page_tab must be contiguous"):
        rg.kv8_append(c, k, k, torch.zeros((2, 3), dtype=I32).t(), n)
    bad = c._replace(k_scale=c.k_scale.double())
    with pytest.raises(TypeError, match="k_scale"):
        rg.kv8_append(bad, k, k, tab, n)
    with pytest.raises(ValueError, match="cache.v must have shape"):
        rg.kv8_append(c._replace(v=c.v[:3]), k, k, tab, n)
    with pytest.raises(ValueError, match="multiple of 16"):
        rg.Kv8Cache.empty(4, 2, 64, 24, device="cpu")
    for page, hd, what in ((48, 64, "power of two"), (2048, 64, "at most 1024"), (16, 96, "head_dim")):
        with pytest.raises(ValueError, match=what):
            rg.Kv8Cache.empty(4, 2, hd, page, device="cpu")


def test_attention_refuses():
    import paper_2606_02218_amd as rg
    c, q = _cache(), _zeros(3, 4, 64)
    tab, n = torch.zeros((3, 2), dtype=I32), torch.ones(3, dtype=I32)
    with pytest.raises(TypeError, match="GPU memory"):
        rg.kv8_attention(c, q, tab, n)
    with pytest.raises(ValueError, match="q must have shape"):
        rg.kv8_attention(c, _zeros(3, 4, 128), tab, n)
    with pytest.raises(ValueError, match="multiple of 2 heads"):
        rg.kv8_attention(c, _zeros(3, 5, 64), tab, n)
    with pytest.raises(ValueError, match="max_len"):
        rg.kv8_attention(c, q, tab, n, max_len=0)
    with pytest.raises(TypeError, match="out must have dtype"):
        rg.kv8_attention(c, q, tab, n, out=q.float())
    with pytest.raises(ValueError, match="out must be contiguous"):
        rg.kv8_attention(c, q, tab, n, out=_zeros(3, 64, 4).transpose(1, 2))


def _abi():
    import paper_2606_02218_amd._kv8 as m
    lib = m._library()
    cache = dict(k=4096, v=8192, k_scale=64, v_scale=128, pages=8, n_kv=2, head_dim=64, page_tokens=16)
    batch = dict(page_tab=256, tab_rows=3, tab_stride=4, tab_row=None, seq_off=None, seq_len=512, n_seqs=3, rows=3)
    return m, lib, cache, batch


def test_packed_arguments_are_the_structures():
    import paper_2606_02218_amd._kv8 as m
    assert m._CACHE(*range(1, 9)) == bytes(m.rg_kv8_cache(*range(1, 9)))
    assert m._BATCH(*range(1, 9)) == bytes(m.rg_kv8_batch(*range(1, 9)))


@pytest.mark.parametrize("change,code,msg", [
    (dict(k=None), -1, "NULL cache"), (dict(v=8200), -1, "aligned"), (dict(pages=0), -1, "pages"),
    (dict(n_kv=0), -1, "n_kv"), (dict(head_dim=96), -4, "head_dim"), (dict(page_tokens=24), -4, "page_tokens"),
    (dict(page_tokens=2048), -4, "page_tokens"), (dict(pages=1 << 31), -4, "blocks"),
    (dict(pages=1 << 26, page_tokens=1024), -4, "blocks"),
    (dict(rows=-1), -1, "out of range"), (dict(page_tab=None), -1, "page_tab"), (dict(seq_len=None), -1, "seq_len"),
    (dict(tab_stride=0), -1, ">= 1"), (dict(rows=4), -1, "rows must equal"), (dict(n_seqs=0, rows=3, seq_off=16), -1, ">= 1"),
    (dict(tab_stride=1 << 27), -1, "2^30"),
])
def test_library_refuses_caches_and_batches(change, code, msg):
    m, lib, cache, batch = _abi()
    c = m.rg_kv8_cache(**{**cache, **{a: b for a, b in change.items() if a in cache}})
    b = m.rg_kv8_batch(**{**batch, **{a: x for a, x in change.items() if a in batch}})
    app = lib.rg_kv8_append(C.byref(c), C.byref(b), 1, 16, 128, 64, 32, 128, 64, None, 0, 0, None, 0, 0, 0, None, None, 0, 0,
                            0, None)
    assert app == code and msg in lib.rg_last_error().decode(), lib.rg_last_error()
    att = lib.rg_kv8_attention(C.byref(c), C.byref(b), 1, 16, 256, 64, 4, 32, 0.125, 64, None, 0, None)
    assert att == code and msg in lib.rg_last_error().decode(), lib.rg_last_error()


def test_library_refuses_the_rest():
    m, lib, cache, batch = _abi()
    c, b = m.rg_kv8_cache(**cache), m.rg_kv8_batch(**batch)

    def err():
        return lib.rg_last_error().decode()

    def app(dtype=1, k=16, q=None, qo=None, q_row=256, n_q=4, cos=None, n_pos=0, rot=0, layout=0):
        return lib.rg_kv8_append(C.byref(c), C.byref(b), dtype, k, 128, 64, 32, 128, 64, q, q_row, 64, qo, 256, 64, n_q,
                                 cos, cos, n_pos, rot, layout, None)

    assert app(dtype=2) == -1 and "dtype" in err()
    assert app(k=None) == -1 and "NULL k" in err()
    assert app(q=16) == -1 and "q_out" in err()
    assert app(q=16, qo=16, q_row=512) == -1 and "strides" in err()
    assert app(q=16, qo=16, n_q=3) == -1 and "multiple" in err()
    assert app(rot=32) == -1 and "table" in err()
    assert app(rot=33, cos=16, n_pos=4) == -1 and "rot_dim" in err()
    assert app(rot=66, cos=16, n_pos=4) == -1 and "rot_dim" in err()
    assert app(rot=32, cos=16, n_pos=0) == -1 and "n_pos" in err()
    assert app(rot=32, cos=16, n_pos=4, layout=2) == -1 and "layout" in err()
    assert lib.rg_kv8_append(None, C.byref(b), 1, 16, 0, 0, 16, 0, 0, None, 0, 0, None, 0, 0, 0, None, None, 0, 0, 0, None) == -1

    def att(dtype=1, q=16, n_q=4, out=32, scale=0.125, max_len=64, scratch=None, nbytes=0):
        return lib.rg_kv8_attention(C.byref(c), C.byref(b), dtype, q, 256, 64, n_q, out, scale, max_len, scratch, nbytes, None)

    assert att(dtype=3) == -1 and "dtype" in err()
    assert att(n_q=3) == -1 and "multiple" in err()
    assert att(n_q=2 * 129) == -4 and "128" in err()
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert att(scale=scale) == -1 and "scale" in err()
    assert att(max_len=0) == -1 and "max_len" in err()
    assert att(q=None) == -1 and "NULL q" in err()
    assert att(out=40) == -1 and "aligned" in err()
    need = lib.rg_kv8_attention_scratch(4, 2, 64, 3, 3, 0, 4096)
    assert need > 0 and att(max_len=4096, scratch=1 << 20, nbytes=need - 1) == -1 and "scratch" in err()
    assert lib.rg_kv8_attention_scratch(4, 2, 64, 0, 0, 0, 64) == 0
    assert lib.rg_kv8_attention_scratch(5, 2, 64, 1, 1, 0, 64) < 0
    assert lib.rg_kv8_attention_scratch(4, 2, 64, 3, 3, 0, 0) < 0

    def rope(dtype=1, x=16, x_row=64, y=32, y_row=64, pos=16, rows=2, heads=1, hd=64, n_pos=4, rot=64, layout=0):
        return lib.rg_rope(dtype, x, x_row, 64, y, y_row, 64, pos, rows, heads, hd, 16, 16, n_pos, rot, layout, 0, None)

    for change, msg in ((dict(dtype=5), "dtype"), (dict(x=None), "NULL"), (dict(pos=None), "NULL"), (dict(rows=-1), "negative"),
                        (dict(hd=63), "odd"), (dict(rot=0), "rot_dim"), (dict(rot=66), "rot_dim"), (dict(n_pos=0), "n_pos"),
                        (dict(layout=-1), "layout"), (dict(y=16, y_row=128), "overlaps")):
        assert rope(**change) == -1 and msg in err(), (change, err())
    assert rope(rows=0) == 0 and rope(heads=0) == 0
    for a, msg in (((0, 64, 1e4, 0, 1, 0, 1, 32), "n_pos"), ((4, 3, 1e4, 0, 1, 0, 1, 32), "odd"), ((4, 64, 0.0, 0, 1, 0, 1, 32), "theta"),
                   ((4, 64, 1e4, 4, 1, 0, 1, 32), "scaling"), ((4, 64, 1e4, 1, 0.5, 0, 1, 32), "factor"),
                   ((4, 2, 1e4, 2, 2, 0, 1, 32), "rot_dim >= 4"), ((4, 64, 1e4, 3, 2, 0, 1, 32), "length"),
                   ((4, 64, 1e4, 3, 2, 4096, 32, 32), "slow < fast")):
        assert lib.rg_rope_table(16, 16, *a, None) == -1 and msg in err(), (a, err())
