"""Rotary positions against the float64 oracle: every layout, part and type,
strides and alignments, gradients, positions outside the table, scaled tables."""
import numpy as np
import pytest
import torch

from kv8_helpers import BF16, F32, UNIT, dev, host, rounded
from oracle import kv8

pytestmark = pytest.mark.gpu


def _table(rng, n_pos, m):
    a = rng.uniform(-np.pi, np.pi, (n_pos, m))
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def _bound(x, cos, sin, layout, dtype, ref):
    """Two products and a sum in fp32 (each product's and the sum's rounding at most 2^-24 of |a c| + |b s|), then the
    output's own rounding."""
    mag = kv8.rotate(np.abs(x), np.abs(cos), -np.abs(sin), layout)       # |a c| + |b s| in the first of a pair
    mag2 = kv8.rotate(np.abs(x), np.abs(cos), np.abs(sin), layout)       # and in the second
    big = np.maximum(np.abs(mag), np.abs(mag2))
    return 3 * 2.0 ** -24 * big + UNIT[dtype] * (np.abs(ref) + 3 * 2.0 ** -24 * big)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rows,heads,hd,rot", [(1, 1, 64, 64), (7, 12, 128, 128), (129, 3, 128, 64), (5, 28, 128, 96),
                                               (33, 2, 80, 80), (9, 5, 80, 22), (4, 3, 6, 2), (3, 2, 256, 250), (2, 9, 64, 8)])
def test_turns_and_turns_back(dtype, layout, rows, heads, hd, rot):
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(rows * 1000 + rot)
    x = rounded(rng.normal(0, 2, (rows, heads, hd)), dtype)
    cos, sin = _table(rng, 50, rot // 2)
    pos = rng.integers(0, 50, rows).astype(np.int32)
    c, s, p, xd = dev(cos), dev(sin), dev(pos), dev(x, dtype)
    for inverse in (False, True):
        ref = kv8.rotate(x, cos[pos], sin[pos], layout, inverse)
        y = rg.rope(xd, p, c, s, layout=layout, inverse=inverse)
        assert y.dtype == dtype and y.shape == xd.shape
        err = np.abs(host(y) - ref)
        assert np.all(err <= _bound(x, cos[pos], sin[pos], layout, dtype, ref)), err.max()
        assert torch.equal(y[..., rot:], xd[..., rot:])
        # in place, and into a given tensor
        z = xd.clone()
        assert rg.rope(z, p, c, s, layout=layout, inverse=inverse, out=z) is z and torch.equal(z, y)
        into = torch.full_like(xd, 7.0)
        rg.rope(xd, p, c, s, layout=layout, inverse=inverse, out=into)
        assert torch.equal(into, y)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_strided_and_unaligned_views(dtype, layout):
    """Heads of a fused projection, transposed orders and views that start at odd elements."""
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(5)
    cos, sin = _table(rng, 40, 32)
    pos = rng.integers(0, 40, 11).astype(np.int32)
    c, s, p = dev(cos), dev(sin), dev(pos)
    base = dev(rng.normal(size=(20 * 11 * 9 * 64,)).astype(np.float32), dtype)
    views = [base[:11 * 9 * 64].view(11, 9, 64)[:, 2:7], base[1:1 + 11 * 9 * 64].view(11, 9, 64)[:, 4:],
             base[:9 * 11 * 64].view(9, 11, 64).transpose(0, 1), base[3:3 + 11 * 5 * 67].view(11, 5, 67)[..., 3:],
             base[:11 * 700].view(11, 700)[:, 8:8 + 5 * 128].unflatten(1, (5, 128))[..., :64]]
    for x in views:
        want = rg.rope(x.contiguous(), p, c, s, layout=layout)
        ref = kv8.rotate(host(x), cos[pos], sin[pos], layout)
        assert np.all(np.abs(host(want) - ref) <= _bound(host(x), cos[pos], sin[pos], layout, dtype, ref))
        assert torch.equal(rg.rope(x, p, c, s, layout=layout), want)
        out = torch.zeros(base.numel(), dtype=dtype, device="cuda").as_strided(x.shape, x.stride(), x.storage_offset())
        assert torch.equal(rg.rope(x, p, c, s, layout=layout, out=out), want)
        around = base.clone()
        z = around.as_strided(x.shape, x.stride(), x.storage_offset())
        rg.rope(z, p, c, s, layout=layout, out=z)
        mask = torch.zeros_like(around, dtype=torch.bool)
        mask.as_strided(x.shape, x.stride(), x.storage_offset()).fill_(True)
        assert torch.equal(z, want) and torch.equal(around[~mask], base[~mask])      # nothing else is touched


def test_gradient():
    """The turn back is the gradient: against the formula (its transpose) and against differences."""
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(6)
    x, g = (rounded(rng.normal(size=(3, 2, 16)), F32) for _ in range(2))
    cos, sin = _table(rng, 9, 6)
    cos *= 1.25                                   # an amplitude, as the scaled tables have
    sin *= 1.25
    pos = np.array([0, 8, 3], np.int32)
    c, s, p = dev(cos), dev(sin), dev(pos)
    for layout in ("half", "interleaved"):
        grad = host(rg.rope(dev(g, F32), p, c, s, layout=layout, inverse=True))
        assert np.all(np.abs(grad - kv8.rotate(g, cos[pos], sin[pos], layout, inverse=True)) <= 2.0 ** -22 * 8)
        step = 2.0 ** -3                          # the map is linear: any step, rounding / step stays small
        for i in rng.choice(x.size, 24, replace=False):
            d = np.zeros(x.size)
            d[i] = step
            up = host(rg.rope(dev(x + d.reshape(x.shape), F32), p, c, s, layout=layout))
            down = host(rg.rope(dev(x - d.reshape(x.shape), F32), p, c, s, layout=layout))
            diff = ((up - down) * g).sum() / (2 * step)
            # two values of a pair change; each of up and down rounds at 3 * 2^-24 (|x| + step) * 1.25 * 2
            slack = 2 * 2 * 3 * 2.0 ** -24 * (np.abs(x).max() + step) * 2.5 * np.abs(g).max() / (2 * step) + 2.0 ** -20
            assert abs(diff - grad.reshape(-1)[i]) <= slack


def test_positions_outside_the_table_and_special_values():
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(7)
    cos, sin = _table(rng, 10, 16)
    x = rng.normal(size=(6, 3, 64)).astype(np.float32)
    x[1, 0, 3], x[1, 1, 40], x[2, 0, 20] = np.nan, np.inf, -np.inf
    pos = np.array([-1, 0, 9, 10, 2 ** 31 - 1, -2 ** 31], np.int32)
    for dtype in (BF16, F32):
        y = host(rg.rope(dev(x, dtype), dev(pos), dev(cos), dev(sin)))
        for r in (0, 3, 4, 5):
            assert np.all(np.isnan(y[r, :, :32])) and np.array_equal(y[r, :, 32:], rounded(x[r, :, 32:], dtype))
        ok = np.array([1, 2])
        with np.errstate(invalid="ignore"):
            ref = kv8.rotate(rounded(x[ok], dtype), cos[pos[ok]], sin[pos[ok]])
        assert np.array_equal(np.isnan(y[ok]), np.isnan(ref)) and np.array_equal(np.isinf(y[ok]), np.isinf(ref))
    assert rg.rope(dev(x[:0]), dev(pos[:0]), dev(cos), dev(sin)).shape == (0, 3, 64)
    assert rg.rope(dev(x[:, :0]), dev(pos), dev(cos), dev(sin)).shape == (6, 0, 64)


@pytest.mark.parametrize("scaling,kw", [(None, {}), ("linear", dict(factor=4.0)), ("base", dict(factor=8.0)),
                                        ("bands", dict(factor=4.0, length=4096.0)),
                                        ("bands", dict(factor=16.0, length=2048.0, slow=2.0, fast=20.0))])
@pytest.mark.parametrize("n_pos,rot,theta", [(1, 64, 1e4), (700, 128, 1e6), (40000, 20, 1e4)])
def test_tables(scaling, kw, n_pos, rot, theta):
    """One rounding to fp32 of values in 64 bits; the angle itself (up to 4e4) is good to 1e-11."""
    import paper_2606_02218_amd as rg
    c, s = rg.rope_table(n_pos, rot, theta, scaling=scaling, **kw)
    w, amp = kv8.frequencies(rot, theta, scaling, **kw)
    a = np.arange(n_pos)[:, None] * w
    assert c.shape == s.shape == (n_pos, rot // 2) and c.dtype == F32
    for got, ref in ((c, amp * np.cos(a)), (s, amp * np.sin(a))):
        assert np.all(np.abs(host(got) - ref) <= 2.0 ** -24 * np.abs(ref) + 1e-10)


def test_far_elements_and_other_streams():
    """Row strides that pass 2^31 elements; a stream of the caller's."""
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(8)
    cos, sin = _table(rng, 4, 32)
    big = torch.empty(3 * 1_200_000_000, dtype=BF16, device="cuda")
    x = big.as_strided((3, 2, 64), (1_199_999_000, 64, 1))
    x.copy_(dev(rng.normal(size=(3, 2, 64)).astype(np.float32), BF16))
    p, c, s = dev(np.array([1, 2, 3], np.int32)), dev(cos), dev(sin)
    want = rg.rope(x.contiguous(), p, c, s)
    assert torch.equal(rg.rope(x, p, c, s), want)
    rg.rope(x, p, c, s, out=x)
    assert torch.equal(x.contiguous(), want)
    del big, x
    st = torch.cuda.Stream()
    xs = torch.randn(1000, 12, 64, device="cuda")
    ps = torch.zeros(1000, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    y = rg.rope(xs, ps, c, s, stream=st)
    st.synchronize()
    assert torch.equal(y, rg.rope(xs, ps, c, s))
