"""An append whose query output overlaps its keys, values or queries is refused by
the library before any device work, and views that merely lie among one another are
not (CPU only; the addresses are stand-ins that nothing reads)."""
import ctypes as C
import itertools
import os

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2606_02218_amd", "librollout.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="library not built")
HD = 64


@pytest.fixture(scope="module")
def call():
    import torch
    if torch.cuda.is_available():
        pytest.skip("stand-in addresses: not where a launch could run")
    import paper_2606_02218_amd._kv8 as m
    lib = m._library()

    def f(rows, n_kv, n_q, k, v, q, out, dtype=1):
        """Views (element, row stride, head stride) of one buffer; the error, or "" where the call got to its launch."""
        eb = 2 if dtype == 1 else 4
        c = m.rg_kv8_cache(4096, 8192, 64, 128, 8, n_kv, HD, 16)
        b = m.rg_kv8_batch(256, rows, 4, None, None, 512, rows, rows)
        k, v, q, out = (((1 << 30) + eb * x[0], *x[1:]) for x in (k, v, q, out))
        assert lib.rg_kv8_append(C.byref(c), C.byref(b), dtype, *k, *v, *q, *out, n_q, None, None, 0, 0, 0, None) < 0
        err = lib.rg_last_error().decode()
        return err if "overlaps" in err else ""
    return f


def _elements(rows, heads, view):
    at, row, head = view
    return at + (np.arange(rows)[:, None, None] * row + np.arange(heads)[:, None] * head + np.arange(HD)).ravel()


def test_parts_of_one_projection(call):
    """[rows, q | k | v], in place and beside; heads in turn (q, k, v of each head side by side); heads first."""
    for rows, dtype in itertools.product((1, 2, 3, 700), (0, 1)):
        n_kv, n_q = 2, 6
        R = (n_q + 2 * n_kv) * HD
        q, k, v = (0, R, HD), (n_q * HD, R, HD), ((n_q + n_kv) * HD, R, HD)
        dense = (n_q * HD, HD)
        assert call(rows, n_kv, n_q, k, v, q, q, dtype) == ""
        assert call(rows, n_kv, n_q, k, v, q, (rows * R, *dense), dtype) == ""
        assert "k or v" in call(rows, n_kv, n_q, k, v, q, (rows * R - 1, *dense), dtype)
        assert "k or v" in call(rows, n_kv, n_q, k, v, q, k, dtype)
        assert "k or v" in call(rows, n_kv, n_q, k, v, q, (2 * HD, R, HD), dtype)     # two heads too far
        assert "k or v" in call(rows, n_kv, n_q, (rows * R, *dense), v, q, v, dtype)
        far = (9 * rows * R, 2 * n_kv * HD, HD), (9 * rows * R + n_kv * HD, 2 * n_kv * HD, HD)
        assert "without being q" in call(rows, n_kv, n_q, *far, q, (8, R, HD), dtype)
        assert "without being q" in call(rows, n_kv, n_q, *far, q, (R * (rows - 1) + HD, *dense), dtype)
        beside = call(rows, n_kv, n_q, *far, q, (n_q * HD, R, HD), dtype)               # its last heads in the next row
        assert "without being q" in beside if rows > 1 else beside == ""
        # each head's q, k and v side by side
        S = 3 * HD
        assert call(rows, 4, 4, (HD, 4 * S, S), (2 * HD, 4 * S, S), (0, 4 * S, S), (0, 4 * S, S), dtype) == ""
        assert "k or v" in call(rows, 4, 4, (HD, 4 * S, S), (2 * HD, 4 * S, S), (0, 4 * S, S), (1, 4 * S, S), dtype)
        # heads first
        H = rows * HD
        assert call(rows, n_kv, n_q, (n_q * H, HD, H), ((n_q + n_kv) * H, HD, H), (0, HD, H), (0, HD, H), dtype) == ""
        assert "k or v" in call(rows, n_kv, n_q, (n_q * H, HD, H), ((n_q + n_kv) * H, HD, H), (0, HD, H), (H, HD, H), dtype)


def test_against_the_elements_themselves(call):
    """Views in step with one another at places of every kind, against their lists of elements."""
    rng = np.random.default_rng(1)
    hits = 0
    for _ in range(400):
        rows, n_kv = int(rng.integers(1, 5)), int(rng.integers(1, 4))
        n_q = n_kv * int(rng.integers(1, 4))
        row = int(rng.choice([HD, 5 * HD, 9 * HD + 8, 14 * HD, 40 * HD]))
        view = lambda: (int(rng.integers(0, 50 * HD)), row, int(rng.choice([HD, 2 * HD, 3 * HD + 8, 7 * HD])))  # noqa: E731
        k, v, q, out = view(), view(), view(), view()
        o = _elements(rows, n_q, out)
        kv = np.concatenate([_elements(rows, n_kv, k), _elements(rows, n_kv, v)])
        want = "k or v" if np.intersect1d(o, kv).size else "without" if q != out and np.intersect1d(o, _elements(rows, n_q, q)).size else ""
        got = call(rows, n_kv, n_q, k, v, q, out)
        assert (want in got) if want else got == "", (rows, n_kv, n_q, k, v, q, out, got, want)
        hits += bool(want)
    assert 50 < hits < 350
