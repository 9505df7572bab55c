"""Calls of more work than one launch's 2^32 threads, and scales past what fp32
holds of them, are refused by the library before any device work (CPU only; the
addresses are stand-ins that nothing reads)."""
import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2606_02218_amd", "librollout.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="library not built")


REFUSED = ("invalid configuration argument", "invalid argument")


def _call(n_kv, rows, seqs):
    """(library, cache, batch) of rows in `seqs` sequences (None: one row a sequence)."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("stand-in addresses: not where a launch could run")
    import paper_2606_02218_amd._kv8 as m
    n = rows if seqs is None else seqs
    return (m._library(), m.rg_kv8_cache(4096, 8192, 64, 128, 8, n_kv, 64, 16),
            m.rg_kv8_batch(256, n, 4, None, None if seqs is None else 1024, 512, n, rows))


# workgroups of 256 threads: (row, kv head) of single rows; (128-row tile or sequence, kv head) of runs
@pytest.mark.parametrize("n_kv,rows,seqs", [(1, 1 << 24, None), (1, (1 << 28) - 1, None), (64, 1 << 18, None), (8, 1 << 28, None),
                                            (1 << 20, 17, 20), (512, 1 << 22, 3), (1 << 23, 100, 3)])
def test_attention_past_a_launch_is_refused(n_kv, rows, seqs):
    lib, c, b = _call(n_kv, rows, seqs)
    assert lib.rg_kv8_attention(C.byref(c), C.byref(b), 1, 16, 64, 64, n_kv, 32, 0.125, 64, 1 << 20, 1 << 62, None) == -3
    assert lib.rg_last_error().decode().split(": ")[1] in REFUSED


# four waves a workgroup: (block of 16 tokens, kv head, keys or values), then the query rows
@pytest.mark.parametrize("n_kv,rows,seqs,q", [(1, 1 << 25, None, False), (8, 1 << 22, None, False), (1, (3 << 24) - 1, None, True),
                                              (1 << 23, 5, 3, False), (64, 1 << 23, 3, False), (1, 1 << 28, None, False)])
def test_appends_past_a_launch_are_refused(n_kv, rows, seqs, q):
    lib, c, b = _call(n_kv, rows, seqs)
    x = (16, 64, 64, 16, 64, 64) if q else (None, 0, 0, None, 0, 0)
    assert lib.rg_kv8_append(C.byref(c), C.byref(b), 1, 1 << 40, 64, 64, 1 << 41, 64, 64, *x, n_kv, None, None, 0, 0, 0, None) == -3
    assert lib.rg_last_error().decode().split(": ")[1] in REFUSED


def test_scales_whose_base_two_form_is_infinite_are_refused():
    lib, c, b = _call(2, 3, None)
    for scale in (2.4e38, 3.4e38):
        assert lib.rg_kv8_attention(C.byref(c), C.byref(b), 1, 16, 128, 64, 4, 32, scale, 64, None, 0, None) == -1
        assert "scale must be" in lib.rg_last_error().decode()
