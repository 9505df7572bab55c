"""Appends to the 8-bit cache against the float64 oracle: codes and scales bit
for bit where nothing is turned, within a code's half step where keys are, over
types, heads, pages, odd runs, strides and everything a batch may hold."""
import numpy as np
import pytest
import torch

from kv8_helpers import BF16, F32, UNIT, Batch, dev, host, offsets, rounded
from oracle import kv8

pytestmark = pytest.mark.gpu


def _same(got, want):
    for g, w, what in zip(got, want, ("k", "k_scale", "v", "v_scale")):
        if g.dtype == np.uint8:
            assert np.array_equal(g, w), (what, int((g != w).sum()), g.size)
        else:
            assert np.array_equal(g, w), what


RUNS = [([1, 1, 1], [0, 5, 31]), ([16, 1, 33], [0, 15, 16]), ([3, 0, 17, 50], [13, 7, 31, 0]),
        ([64], [0]), ([1] * 20, list(range(20))), ([100, 2], [1, 127])]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n_kv,hd,page", [(2, 128, 16), (3, 64, 64), (1, 128, 1024), (12, 64, 32)])
@pytest.mark.parametrize("new,old", RUNS)
def test_codes_and_scales_bit_for_bit(dtype, n_kv, hd, page, new, old):
    import paper_2606_02218_amd as rg
    b = Batch(old, n_kv, hd, page, capacity=max(a + c for a, c in zip(new, old)), seed=hd + page + len(new))
    rows = sum(new)
    gain = np.exp(b.rng.normal(0, 1.0, (rows, 1, 1)))             # rows of several sizes: scales grow on the way
    k, v = (rounded(b.rng.normal(size=(rows, n_kv, hd)) * gain, dtype) for _ in range(2))
    at = np.cumsum([0] + new)
    for s in range(len(new)):
        b.k[s].append(k[at[s]:at[s + 1]])
        b.v[s].append(v[at[s]:at[s + 1]])
    want = b.image()
    off = None if set(new) == {1} else offsets(new)
    rg.kv8_append(b.cache, dev(k, dtype), dev(v, dtype), dev(b.tab), dev(b.lengths()), off)
    _same(b.snapshot(), want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("hd,rot", [(128, 128), (128, 64), (64, 64), (64, 20), (128, 6)])
@pytest.mark.parametrize("new,old", [([1, 1], [0, 30]), ([40, 7], [9, 0])])
def test_turned_keys_and_queries(dtype, layout, hd, rot, new, old):
    """A stored key is within half a code step of the turned key; the turn's own fp32 error (3 roundings of 2^-24 of
    |a c| + |b s|) adds to it.  Block scales are those of the oracle: no largest magnitude here lies within that error
    of a power's border."""
    import paper_2606_02218_amd as rg
    b = Batch(old, 2, hd, 32, capacity=80, seed=rot + hd)
    rows = sum(new)
    k, v, q = (rounded(b.rng.normal(size=(rows, h, hd)), dtype) for h in (2, 2, 6))
    a = b.rng.uniform(-3, 3, (80, rot // 2))
    cos, sin = np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)
    pos = np.concatenate([np.arange(o, o + n) for n, o in zip(new, old)])
    turned = kv8.rotate(k, cos[pos], sin[pos], layout)
    slip = 3 * 2.0 ** -24 * 2 * np.abs(k).max()
    at = np.cumsum([0] + new)
    for s in range(len(new)):
        for x, seq in ((turned, b.k[s]), (v, b.v[s])):
            seq.append(x[at[s]:at[s + 1]])
    want = b.image()
    off = None if set(new) == {1} else offsets(new)
    qd = dev(q, dtype)
    out = rg.kv8_append(b.cache, dev(k, dtype), dev(v, dtype), dev(b.tab), dev(b.lengths()), off, q=qd, cos=dev(cos),
                        sin=dev(sin), layout=layout)
    got = b.snapshot()
    assert np.array_equal(got[1], want[1]) and np.array_equal(got[3], want[3]) and np.array_equal(got[2], want[2])
    for s in range(len(new)):
        n = old[s] + new[s]
        held = b.logical(s, n, True)[old[s]:]
        y = turned[at[s]:at[s + 1]]
        scale = np.repeat(b.k[s].scale, 16, 0)[old[s]:n, :, None]
        step = np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * scale)
        assert np.all(np.abs(held - y) <= step * (1 + 2.0 ** -20) + 2 * slip)
        # tokens that stay: the oracle's
        assert np.array_equal(b.logical(s, n, True)[:old[s]], b.k[s].values()[:old[s]])
    # queries exactly as the standalone rotation leaves them, in place too
    ref = rg.rope(qd, dev(pos.astype(np.int32)), dev(cos), dev(sin), layout=layout)
    assert torch.equal(out, ref)
    rg.kv8_append(b.cache, dev(k, dtype), dev(v, dtype), dev(b.tab), dev(b.lengths()), off, q=qd, cos=dev(cos),
                  sin=dev(sin), layout=layout, q_out=qd)
    assert torch.equal(qd, ref)
    _same(b.snapshot(), got)                                      # the same rows again leave the same


def test_token_by_token_grows_scales():
    """40 single tokens of growing size against the oracle, appended the same way; and what a sequence holds then
    against the values: each requantization rounds by at most half a subnormal step of the scale it rounds to."""
    import paper_2606_02218_amd as rg
    b = Batch([0, 3], 2, 64, 16, capacity=48, seed=4)
    tab = dev(b.tab)
    true = [[], []]
    for i in range(40):
        k, v = (rounded(b.rng.normal(size=(2, 2, 64)) * 1.12 ** i, F32) for _ in range(2))
        for s in range(2):
            b.k[s].append(k[s:s + 1])
            b.v[s].append(v[s:s + 1])
            true[s].append(v[s])
        want = b.image()
        rg.kv8_append(b.cache, dev(k, F32), dev(v, F32), tab, dev(b.lengths()))
        _same(b.snapshot(), want)
    for s, n0 in ((0, 0), (1, 3)):
        got, scale = b.logical(s, n0 + 40, False)[n0:], np.repeat(b.v[s].scale, 16, 0)[n0:n0 + 40, :, None]
        x = np.stack(true[s])
        # first rounding: half a step; later ones: halves of subnormal steps of growing scales, at most twice the last's
        assert np.all(np.abs(got - x) <= 2.0 ** -4 * np.abs(x) + 2 * 2.0 ** -10 * scale)


def test_special_values():
    import paper_2606_02218_amd as rg
    b = Batch([0, 0, 0, 2], 1, 64, 16, capacity=32, seed=9)
    n = [2, 3, 1, 2]
    x = rounded(b.rng.normal(size=(8, 1, 64)), F32)
    x[0, 0, :4] = [np.nan, np.inf, -np.inf, -0.0]
    x[2:5] = 0.0                                                   # a block of zeros
    x[5] = np.nan                                                  # of NaN
    x[6, 0, 0], x[7, 0, 1] = 3.3e38, 1e-38
    at = np.cumsum([0] + n)
    for s in range(4):
        b.k[s].append(x[at[s]:at[s + 1]])
        b.v[s].append(x[at[s]:at[s + 1]])
    want = b.image()
    rg.kv8_append(b.cache, dev(x, F32), dev(x, F32), dev(b.tab), dev(b.lengths()), offsets(n))
    _same(b.snapshot(), want)


def test_strided_and_unaligned_views():
    import paper_2606_02218_amd as rg
    new, old = [20, 3], [5, 0]
    rng = np.random.default_rng(3)
    for dtype in (BF16, F32):
        base = dev(rng.normal(size=23 * 10 * 128 + 16).astype(np.float32), dtype)
        fused = base[:23 * 10 * 128].view(23, 10, 128)
        odd = base[1:1 + 23 * 10 * 128].view(23, 10, 128)
        swapped = base[:10 * 23 * 128].view(10, 23, 128).transpose(0, 1)
        a = rng.uniform(-3, 3, (40, 64))
        cos, sin = dev(np.cos(a).astype(np.float32)), dev(np.sin(a).astype(np.float32))
        for src in (fused, odd, swapped):
            q, k, v = src[:, :6], src[:, 6:8], src[:, 8:]
            got = []
            for x in ((q, k, v), (q.contiguous(), k.contiguous(), v.contiguous())):
                b = Batch(old, 2, 128, 16, capacity=40, seed=1)
                ln = dev((b.lengths() + np.array(new)).astype(np.int32))
                out = rg.kv8_append(b.cache, x[1], x[2], dev(b.tab), ln, offsets(new), q=x[0], cos=cos, sin=sin)
                got.append([out.cpu()] + b.snapshot())
            assert torch.equal(got[0][0], got[1][0])
            _same(got[0][1:], got[1][1:])


def test_padding_rows_foreign_rows_and_lost_pages():
    """Sequences shorter than their rows, empty ones, rows behind the last sequence, a table picked by tab_row, page
    ids that are none of the pool's and positions past the table: nothing but the rest is written."""
    import paper_2606_02218_amd as rg
    b = Batch([0, 4, 0, 0], 2, 64, 16, capacity=64, seed=11)
    new = [5, 3, 0, 2]                                              # sequence 0 holds only 2 tokens after the call
    k = rounded(b.rng.normal(size=(14, 2, 64)), BF16)               # 10 rows and 4 of nobody
    q = dev(b.rng.normal(size=(14, 4, 64)).astype(np.float32), BF16)
    cos, sin = np.ones((64, 32), np.float32), np.zeros((64, 32), np.float32)    # turned by nothing: exact
    for s, rows in ((0, k[3:5]), (1, k[5:8]), (3, k[8:10])):
        b.k[s].append(rows)
        b.v[s].append(rows)
    length = np.array([2, 7, 0, 2], np.int32)
    order = np.array([3, 0, 2, 1])                                  # the table's rows in another order
    tab = np.zeros((5, b.width), np.int32)
    tab[order] = b.tab
    tab[4] = -1
    want = b.image()
    q_out = torch.full_like(q, 5.0)
    rg.kv8_append(b.cache, dev(k, BF16), dev(k, BF16), dev(tab), dev(length), offsets(new), q=q, q_out=q_out,
                  cos=dev(cos), sin=dev(sin), tab_row=dev(order.astype(np.int32)))
    _same(b.snapshot(), want)
    assert torch.all(q_out[:3] == 5.0) and torch.all(q_out[10:] == 5.0) and torch.equal(q_out[3:10], q[3:10])
    # lost pages: each of these drops its rows and writes nowhere
    before = b.snapshot()
    one = dev(k[:4], BF16)
    for table, tr, ln in (([[-1, 0], [b.pages, 0], [2 ** 31 - 1, 0], [-2 ** 31, 0]], None, [1, 1, 1, 1]),
                          ([[0, 0]] * 4, [4, -1, 2 ** 31 - 1, -2 ** 31], [1, 1, 1, 1]),
                          ([[0, 0]] * 4, None, [33, 1000, 2 ** 31 - 1, -5])):
        t = np.array(table, np.int64).astype(np.int32)
        rg.kv8_append(b.cache, one, one, dev(t), dev(np.array(ln, np.int64).astype(np.int32)),
                      tab_row=None if tr is None else dev(np.array(tr, np.int64).astype(np.int32)))
        _same(b.snapshot(), before)
    # runs that end at the largest length there is: no page holds them
    rg.kv8_append(b.cache, one, one, dev(np.array([[0, 0]] * 2, np.int32)), dev(np.array([2 ** 31 - 1, 2 ** 31 - 16], np.int32)),
                  offsets([3, 1]))
    many = dev(np.repeat(k[:4], 30, 0), BF16)
    rg.kv8_append(b.cache, many, many, dev(np.array([[0, 0]], np.int32)), dev(np.array([2 ** 31 - 1], np.int32)), offsets([120]))
    _same(b.snapshot(), before)
    # offsets out of order or out of range reach no row outside the call's
    for off in ([0, 9, 3, 2, 4], [-7, 0, 2, 2, 100], [50, 60, 70, 80, 90]):
        rg.kv8_append(b.cache, one, one, dev(tab), dev(np.array([1, 1, 1, 1], np.int32)), dev(np.array(off, np.int32)),
                      tab_row=dev(np.full(4, 4, np.int32)))
        _same(b.snapshot(), before)
    # a key past the rotary table is NaN, its value as it is
    rg.kv8_append(b.cache, one[:1], one[:1], dev(b.tab[:1]), dev(np.array([3], np.int32)), cos=dev(cos[:2]), sin=dev(sin[:2]))
    assert np.all(np.isnan(b.logical(0, 3, True)[2])) and np.all(np.isfinite(b.logical(0, 3, False)[2]))


def test_empty_calls():
    import paper_2606_02218_amd as rg
    b = Batch([3], 2, 64)
    before = b.snapshot()
    z = torch.zeros(0, 2, 64, device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert rg.kv8_append(b.cache, z, z, torch.zeros(0, 1, dtype=torch.int32, device="cuda"), none) is None
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    rg.kv8_append(b.cache, z, z, dev(b.tab), one, torch.zeros(2, dtype=torch.int32, device="cuda"))
    _same(b.snapshot(), before)
