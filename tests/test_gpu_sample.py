"""Sampling from given logits and uniform numbers against the float64 oracle."""
import math

import numpy as np
import pytest
import torch

from oracle.draw import Row, weight_slack

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def logits(rng, rows, vocab, kind, dtype):
    z = rng.normal(0, 2.0, (rows, vocab))
    if kind == "peaked":                   # as a decoder's: a few far above the rest
        for r in range(rows):
            at = rng.integers(0, vocab, min(30, vocab))
            z[r, at] = rng.uniform(8, 18) - rng.uniform(0, 9, len(at))
    elif kind == "sharp":
        z[np.arange(rows), rng.integers(0, vocab, rows)] = 30.0
    elif kind == "equal":
        z[:] = 1.25
    elif kind == "few values":
        z = rng.integers(-3, 4, (rows, vocab)) * 0.5
    elif kind == "masked":
        z[rng.random((rows, vocab)) < 0.9] = -np.inf
        z[rng.random((rows, vocab)) < 0.2] = -3.3895314e38
        z[:, vocab // 2] = 1.0
    elif kind == "ascending":
        z = np.sort(z, 1)
    return torch.from_numpy(z).to(dtype).cuda()


def check(z, u, got, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Each row's draw is one that the oracle's sums, moved by no more than the weights' own error, can give."""
    token, lp, kept = (x.cpu().numpy() for x in got)
    z, u = z.double().cpu().numpy(), u.double().cpu().numpy()
    row = lambda x, r: x[r].item() if isinstance(x, torch.Tensor) else x  # noqa: E731
    wide = 0
    for r in range(len(z)):
        t = row(temperature, r)
        s = weight_slack(z[r], t)
        o = Row(z[r], t, row(top_k, r), row(top_p, r), row(min_p, r), 2 * s)
        wide += o.low != o.high
        fits = []
        for n in range(o.low, o.high + 1):
            if token[r] not in o.kept(n):
                fits.append("not kept")
                continue
            a, b = o.span(token[r], n)
            _, want_lp, want_kept = o.logs(token[r], n)
            if t == 0:
                assert token[r] == o.order[0]
                a, b = 0.0, 1.0
            ok = a - 4 * s <= u[r] <= b + 4 * s
            # the sum is off by s, its logarithm so much; the result is rounded once (2^-24)
            near = all(abs(x - y) <= 2 * s + 2.0 ** -24 * abs(y) * 1.01 + 1e-12 for x, y in ((lp[r], want_lp), (kept[r], want_kept)))
            fits.append(ok and near or (a, b, u[r], lp[r], want_lp, kept[r], want_kept, s))
        assert True in fits, (r, token[r], o.low, o.high, fits[:3])
    return wide


KINDS = ["peaked", "flat", "sharp", "equal", "few values", "masked", "ascending"]
SETTINGS = [dict(), dict(temperature=0.6), dict(top_k=1), dict(top_k=20), dict(top_k=300), dict(top_p=0.9), dict(top_p=0.1),
            dict(top_p=0.999), dict(min_p=0.05), dict(min_p=1.0), dict(top_k=50, top_p=0.8, temperature=0.7),
            dict(top_k=40, top_p=0.95, min_p=0.1, temperature=1.3), dict(top_p=0.7, min_p=0.01), dict(top_k=7, min_p=0.3),
            dict(temperature=0.0), dict(temperature=0.0, top_p=0.5)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("vocab", [1, 7, 512, 1000, 5003])
def test_small_vocabularies(dtype, kind, vocab):
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(vocab + len(kind))
    z = logits(rng, 6, vocab, kind, dtype)
    for i, s in enumerate(SETTINGS):
        u = torch.from_numpy(rng.random(6)).cuda()
        if i % 2:
            u = u.float().clamp(max=1 - 2.0 ** -24)
        check(z, u, rg.sample(z, u, **s), **s)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", KINDS)
def test_large_vocabularies(dtype, kind):
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(len(kind))
    z = logits(rng, 5, 151936, kind, dtype)
    for s in SETTINGS:
        u = torch.from_numpy(rng.random(5)).cuda()
        check(z, u, rg.sample(z, u, **s), **s)


def test_largest_vocabulary_and_many_rows():
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(1)
    z = logits(rng, 2, 1 << 20, "peaked", F32)
    for s in (dict(), dict(top_p=0.95), dict(top_k=100, top_p=0.9), dict(min_p=1e-6), dict(top_k=1000000)):
        u = torch.from_numpy(rng.random(2)).cuda()
        check(z, u, rg.sample(z, u, **s), **s)
    z = logits(rng, 700, 900, "peaked", BF16)
    for s in (dict(), dict(top_k=30, top_p=0.9)):
        u = torch.from_numpy(rng.random(700)).cuda()
        check(z, u, rg.sample(z, u, **s), **s)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["peaked", "flat", "equal", "few values"])
@pytest.mark.parametrize("rows,vocab", [(3, 1024), (3, 1025), (4, 4097), (4, 16384), (4, 16385), (255, 4099), (257, 4099)])
def test_both_sides_of_each_choice(rows, vocab, kind, dtype):
    """Lists and histograms, a workgroup a row and several, k by segments, strips and tokens."""
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(rows + vocab)
    z = logits(rng, rows, vocab, kind, dtype)
    for s in (dict(top_p=0.9), dict(min_p=0.02), dict(top_p=0.8, min_p=0.02), dict(top_k=4), dict(top_k=5, top_p=0.9),
              dict(top_k=vocab // 128), dict(top_k=vocab // 128 + 1, min_p=0.05), dict(top_k=vocab // 64 + 40, top_p=0.95),
              dict(top_k=vocab - 1)):
        u = torch.from_numpy(rng.random(rows)).cuda()
        check(z, u, rg.sample(z, u, **s), **s)


@pytest.mark.parametrize("rows,vocab", [(30, 4200), (300, 4200), (260, 20000)])
def test_rows_that_go_different_ways(rows, vocab):
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(rows)
    z = logits(rng, rows, vocab, "flat", BF16)
    u = torch.from_numpy(rng.random(rows)).cuda()
    some = lambda p, a, b: torch.from_numpy(np.where(rng.random(rows) < p, a, b))  # noqa: E731
    s = dict(temperature=some(0.1, 0.0, rng.uniform(0.1, 2, rows)).float().cuda(),
             top_k=some(0.5, 0, rng.integers(1, 4400, rows)).int().cuda(),
             top_p=some(0.4, 1.0, rng.uniform(0.05, 1, rows)).float().cuda(),
             min_p=some(0.5, 0.0, rng.uniform(0, 0.6, rows)).float().cuda())
    check(z, u, rg.sample(z, u, **s), **s)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab", [(255, 32768), (256, 32768), (256, 32769), (256, 50257)])
def test_rows_with_k_of_their_own_in_larger_vocabularies(rows, vocab, dtype):
    """A workgroup a row up to some size, several past it: half of the rows by top-p or min-p alone."""
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(rows + vocab)
    z = logits(rng, rows, vocab, "peaked", dtype)
    u = torch.from_numpy(rng.random(rows)).cuda()
    k = torch.from_numpy(np.where(rng.random(rows) < 0.5, 0, rng.integers(1, 60, rows))).int().cuda()
    for s in (dict(top_k=k, top_p=0.9), dict(top_k=k, min_p=0.05), dict(top_k=k * 0, top_p=0.5, min_p=0.001)):
        check(z, u, rg.sample(z, u, **s), **s)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_settings_by_row_strides_and_repeats(dtype):
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(4)
    rows, vocab = 40, 3001
    z = logits(rng, rows, vocab, "peaked", dtype)
    u = torch.from_numpy(rng.random(rows)).float().cuda()
    s = dict(temperature=torch.from_numpy(np.where(rng.random(rows) < 0.2, 0.0, rng.uniform(0.3, 2, rows))).float().cuda(),
             top_k=torch.from_numpy(rng.integers(-2, 60, rows)).int().cuda(),
             top_p=torch.from_numpy(np.where(rng.random(rows) < 0.3, 1.0, rng.uniform(-0.1, 1.2, rows))).float().cuda(),
             min_p=torch.from_numpy(np.where(rng.random(rows) < 0.5, -1.0, rng.uniform(0, 0.4, rows))).float().cuda())
    want = rg.sample(z, u, **s)
    check(z, u, want, **s)
    for off in (0, 1, 3, 8):               # rows of a wider matrix, at any alignment
        wide = torch.full((rows, vocab + 13), float("nan"), device="cuda", dtype=dtype)
        wide[:, off:off + vocab] = z
        for a, b in zip(rg.sample(wide[:, off:off + vocab], u, **s), want):
            assert torch.equal(a, b)
    for _ in range(3):
        for a, b in zip(rg.sample(z, u, **s), want):
            assert torch.equal(a, b)
    # one row for every uniform number: rows that share their memory
    one = z[:1].expand(rows, vocab)
    check(one, u, rg.sample(one, u, top_k=20), top_k=20)


def test_more_rows_than_a_launch_takes():
    """Refused before the first kernel: outputs and scratch stay as they were."""
    import ctypes as C

    import paper_2606_02218_amd as rg
    from paper_2606_02218_amd import _draft
    rows = 1 << 23
    z = torch.zeros(1, 1, device="cuda").expand(rows, 1)
    u = torch.zeros(rows, device="cuda")
    lib = _draft._library()
    o = _draft.rg_sample_options(1.0, 0.9, 0.0, 0)
    need = lib.rg_sample_scratch(rows, 1, C.byref(o))
    token, lp, scratch = (torch.full((n,), 77, dtype=torch.int32, device="cuda") for n in (rows, 2 * rows, need // 4))
    rc = lib.rg_sample(0, z.data_ptr(), 0, rows, 1, 0, u.data_ptr(), C.byref(o), token.data_ptr(), lp.data_ptr(),
                       lp.data_ptr() + 4 * rows, scratch.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    assert rc == -3 and b"rg_sample" in lib.rg_last_error()
    torch.cuda.synchronize()
    assert all(bool((x == 77).all()) for x in (token, lp, scratch))
    assert bool((rg.sample(z[1:], u[1:], top_p=0.9)[0] == 0).all())


def test_frequencies():
    """20000 draws from eight tokens: counts within five deviations, both ways of drawing."""
    import paper_2606_02218_amd as rg
    z = torch.tensor([0.0, 1.0, -1.0, 2.0, 0.5, -3.0, 1.5, -0.5], device="cuda")
    n = 20000
    u = (torch.arange(n, device="cuda", dtype=torch.float64) + 0.5) / n
    for s in (dict(), dict(top_k=5), dict(top_p=0.8), dict(min_p=0.1)):
        token = rg.sample(z.expand(n, 8), u, **s)[0].cpu().numpy()
        o = Row(z.double().cpu().numpy(), **s)
        p = np.zeros(8)
        p[o.kept(o.low)] = o.w[o.kept(o.low)] / o.w[o.kept(o.low)].sum()
        assert np.all(np.abs(np.bincount(token, minlength=8) - n * p) <= 1.01)


@pytest.mark.parametrize("s", [dict(), dict(top_k=50), dict(top_p=0.9), dict(top_k=50, top_p=0.9), dict(min_p=0.01)])
def test_the_ends_of_u(s):
    """u = 0 and the largest number below 1: the first and the last token that is kept and has a weight."""
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(9)
    for vocab in (700, 40000):
        z = logits(rng, 3, vocab, "masked", F32)
        z[2] = logits(rng, 1, vocab, "peaked", F32)[0]
        for u in (torch.zeros(3, device="cuda"), torch.full((3,), 1 - 2.0 ** -53, device="cuda", dtype=torch.float64)):
            token = rg.sample(z, u, **s)[0].cpu().numpy()
            for r in range(3):
                o = Row(z[r].double().cpu().numpy(), **s, slack=1e-6)
                first = [o.kept(n)[o.w[o.kept(n)] > 2.0 ** -40] for n in (o.low, o.high)]
                # what weighs less than the sums' steps may or may not be passed
                assert token[r] <= max(x[0] for x in first) if u[0] == 0 else token[r] >= min(x[-1] for x in first)


@pytest.mark.parametrize("s", [dict(), dict(top_k=5), dict(top_p=0.9), dict(min_p=0.1), dict(temperature=0.0)])
def test_rows_that_have_no_answer(s):
    """NaN and infinities, nothing but -inf, u outside [0, 1): token -1 and NaN; the rows beside them as ever."""
    import paper_2606_02218_amd as rg
    inf, nan = math.inf, math.nan
    rng = np.random.default_rng(2)
    z = logits(rng, 10, 1300, "peaked", F32)
    z[1, 700] = nan
    z[2, 1299] = inf
    z[3] = -inf
    z[4, 3] = -nan
    u = torch.tensor([0.5] * 5 + [1.0, -0.1, nan, 0.0, 0.25], device="cuda")
    token, lp, kept = rg.sample(z, u, **s)
    for r in range(1, 8):
        assert token[r] == -1 and lp[r].isnan() and kept[r].isnan(), r
    good = [0, 8, 9]
    check(z[good], u[good], [x[good] for x in (token, lp, kept)], **s)
    t = torch.full((10,), 1.0, device="cuda")
    t[0], t[8] = -1.0, nan
    token = rg.sample(z, u, temperature=t, top_k=3)[0]
    assert token[0] == -1 and token[8] == -1 and token[9] >= 0
    p = torch.full((10,), 0.5, device="cuda")
    p[0] = nan
    assert rg.sample(z, u, top_p=p)[0][0] == -1 and rg.sample(z, u, min_p=p)[0][0] == -1


def test_extreme_temperatures_and_logits():
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(3)
    z = logits(rng, 4, 2000, "flat", F32)
    u = torch.from_numpy(rng.random(4)).cuda()
    for t in (1e-38, 1e-30, 1e-5, 1e30):
        token, lp, kept = rg.sample(z, u, temperature=t)
        if t < 1e-4:
            assert torch.equal(token.long(), z.argmax(1)) and bool((lp == 0).all())
        else:
            check(z, u, (token, lp, kept), temperature=t)
        check(z, u, rg.sample(z, u, temperature=t, top_k=3), temperature=t, top_k=3)
    z = z * 1e37
    check(z, u, rg.sample(z, u, temperature=1e37, top_p=0.9), temperature=1e37, top_p=0.9)
    big = torch.full((2, 700), torch.finfo(F32).min, device="cuda")   # the type's lowest value everywhere
    check(big, u[:2], rg.sample(big, u[:2], top_k=9), top_k=9)
    check(big, u[:2], rg.sample(big, u[:2]))


@pytest.mark.parametrize("vocab", [900, 5000])
@pytest.mark.parametrize("s", [dict(), dict(top_k=3), dict(top_p=0.9), dict(min_p=0.5), dict(top_k=40, top_p=0.5, min_p=0.1)])
def test_the_ends_of_temperature(s, vocab):
    """1 / T past the largest double, and no logit telling from another."""
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(vocab)
    z = logits(rng, 3, vocab, "flat", F32)
    u = torch.from_numpy(rng.random(3)).cuda()
    token, lp, kept = rg.sample(z, u, temperature=5e-324, **s)
    assert torch.equal(token.long(), z.argmax(1)) and bool((lp == 0).all()) and bool((kept == 0).all())
    z[:, :40] = z.amax(1, keepdim=True)    # of equal ones the u-th
    token, lp, kept = rg.sample(z, u, temperature=5e-324)
    for r in range(3):                     # the first 40 and, where it lies behind them, the row's largest itself
        ids = (z[r] == z[r].max()).nonzero().flatten().tolist()
        assert len(ids) in (40, 41) and token[r].item() == ids[int(u[r].item() * len(ids))]
        assert abs(lp[r].item() + np.log(len(ids))) < 2.0 ** -22
    z = logits(rng, 3, vocab, "flat", F32)
    check(z, u, rg.sample(z, u, temperature=1.7e308, **s), temperature=1.7e308, **s)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("t", [1e-300, 1e-40, 1e-33, 1e-29, 1e-6, 1.0, 1e6, 1e29, 1e32, 1e300])
def test_a_largest_logit_of_zero(t, dtype):
    """Nothing tells z / T from z where z is 0: each way of scaling it."""
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(8)
    z = logits(rng, 3, 1500, "flat", dtype)
    z = z - z.amax(1, keepdim=True)
    u = torch.from_numpy(rng.random(3)).cuda()
    for s in (dict(), dict(top_k=30), dict(top_p=0.9), dict(min_p=0.1)):
        got = rg.sample(z, u, temperature=t, **s)
        if 1e-6 <= t:
            check(z, u, got, temperature=t, **s)
        else:
            for r in range(3):             # the u-th of those at the top, or of all that some rule leaves of them
                top = (z[r] == 0).nonzero().flatten().tolist()
                assert got[0][r].item() in top and abs(got[1][r].item() + np.log(len(top))) < 2.0 ** -22
        if 1e-38 <= t <= 1e38:
            row = rg.sample(z, u, temperature=torch.full((3,), t, device="cuda"), **s)
            assert torch.equal(row[0], rg.sample(z, u, temperature=float(np.float32(t)), **s)[0])


@pytest.mark.parametrize("s", [dict(), dict(top_k=20, top_p=0.9)])
def test_graphs_and_streams(s):
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(6)
    z = logits(rng, 9, 20000, "peaked", BF16)
    u = torch.from_numpy(rng.random(9)).float().cuda()
    want = rg.sample(z, u, **s)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = rg.sample(z, u, stream=side, **s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs = []
    for _ in range(2):                     # two graphs, each with scratch of its own
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = rg.sample(z, u, **s)
        graphs.append((g, out))
    for i in range(3):
        u.copy_(torch.from_numpy(rng.random(9)).float())
        want = rg.sample(z, u, **s)
        for g, out in graphs:
            for x in out:
                x.zero_()
            g.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab", [(40, 1025), (300, 5000), (64, 16384), (260, 32000)])
def test_the_same_call_gives_the_same_bits(rows, vocab, dtype):
    """Rows that a workgroup searches by itself, where the sum comes right before the search: many calls, alone and
    beside others, with the oracle's draws."""
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(vocab)
    z = logits(rng, rows, vocab, "peaked", dtype)
    u = torch.from_numpy(rng.random(rows)).cuda()
    full = lambda x, t: torch.full((rows,), x, device="cuda", dtype=t)  # noqa: E731
    k = torch.from_numpy(np.where(rng.random(rows) < 0.5, 0, rng.integers(1, 60, rows))).int().cuda()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in (dict(top_p=0.9, top_k=full(0, torch.int32)), dict(top_p=0.7, min_p=0.02, top_k=full(0, torch.int32)),
              dict(top_p=full(0.8, F32), top_k=k), dict(top_k=40, top_p=0.9)):
        want = rg.sample(z, u, **s)
        check(z, u, want, **s)
        torch.cuda.synchronize()
        got = [rg.sample(z, u, stream=streams[i % 2], **s) for i in range(40)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x in got for a, b in zip(x, want))


# ---------------------------------------------------------------- the sums, as exact as they are said to be
WEIGHT = 2e-12                # a weight's relative error, as rollout.h has it
ONE = 2.0 ** 42               # whole numbers of a weight of 1
ADDED = 64 * 2.0 ** -53       # some 50 additions and products of doubles, each off by half a step


class Sums:
    """A row's weights in 80 bits; where something is cut, the whole numbers that they round to, and how far each can be
    off since the weight is (0 for all but those next to a half)."""

    def __init__(self, z, t, cut):
        z = np.asarray(z, np.longdouble)
        self.w = np.exp((z - z.max()) / np.longdouble(t))
        self.z, self.order = z, np.argsort(-z, kind="stable")
        self.cut, self.value, self.off = cut, self.w, WEIGHT * self.w
        if cut:
            x = self.w * np.longdouble(ONE)
            self.value = np.rint(x)
            self.off = np.maximum(self.value - np.rint(x * (1 - WEIGHT)), np.rint(x * (1 + WEIGHT)) - self.value)

    def spans(self, ids):
        """For ids in order: the shares of u from and to which each is drawn, and how far those can be off.  A share is
        R / (R + S), R the running sum and S what is behind it.  Whole numbers are the same ones wherever they are
        added, so with R off by r and S by s the share is off by (r S + s R) / (R + S)^2.  Uncut rows' weights are taken
        twice, for the sum T and again for the running sum, each time with an error of its own: with R off by r, and T,
        by itself, by e T, R / T is off by (r + e R) / T."""
        v, run, off = self.value[ids], np.cumsum(self.value[ids]), np.cumsum(self.off[ids])
        share = run / run[-1]
        if self.cut:
            slack = (off * (1 - share) + (off[-1] - off) * share) / run[-1]
        else:
            slack = (off + WEIGHT * run) / run[-1]
        return (run - v) / run[-1], share, slack * (1 + 1e-6) + ADDED


def rules(o, z, t):
    """Settings whose kept tokens no error of a sum can change, and those tokens."""
    n = len(z)
    w, order = o.w, o.order
    run = np.cumsum(w[order])
    few = min(20, n)
    yield dict(top_k=few), order[:few]
    many = min(3000, n // 2)
    yield dict(top_k=many), order[:many]
    for k, p in ((0, 0.9), (0, 0.5), (many, 0.8)):        # the border in the middle of a token
        of = run[k - 1] if k else run[-1]
        i = int(np.searchsorted(run, p * of))
        yield dict(top_k=k, top_p=float((run[i] - w[order[i]] / 2) / of)), order[:i + 1]
    values = np.unique(z)[::-1]
    i = np.searchsorted(-values, -(values[0] + t * math.log(0.02)))
    at = (values[i - 1] + values[min(i, len(values) - 1)]) / 2
    yield dict(min_p=float(np.exp((at - values[0]) / np.longdouble(t)))), np.flatnonzero(z >= at)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["flat", "peaked"])
@pytest.mark.parametrize("vocab,rows", [(151936, 3), (16000, 3), (5003, 3), (900, 3), (32000, 5)])
@pytest.mark.parametrize("t", [1.0, 0.7])
def test_draws_turn_where_exact_sums_do(vocab, rows, kind, dtype, t):
    """Uniform numbers just inside both ends of tokens' shares, as near as the weights' stated error lets them be (some
    1e-12, where sums of fp32 weights are 1e-8 off), and the log-probabilities."""
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(vocab)
    z = logits(rng, rows, vocab, kind, dtype)
    host = z.double().cpu().numpy()
    tested = 0
    for r in range(rows):
        plain, cut = Sums(host[r], t, False), Sums(host[r], t, True)
        for o, (s, kept) in [(plain, (dict(), np.arange(vocab)))] + [(cut, x) for x in rules(cut, host[r], t)]:
            ids = np.sort(kept)
            a, b, slack = o.spans(ids)
            good = np.flatnonzero((b - a > 8 * slack) & (o.value[ids] > 0))
            at = np.unique(np.r_[good[:2], good[-2:], rng.choice(good, min(40, len(good)), replace=False)])
            before = np.where(at > 0, slack[np.maximum(at - 1, 0)], 0)
            u = np.r_[(a[at] + before).astype(np.float64), (b[at] - slack[at]).astype(np.float64)]
            ok = (u >= 0) & (u < 1)
            want = np.r_[ids[at], ids[at]][ok]
            got = rg.sample(z[r:r + 1].expand(len(want), vocab), torch.from_numpy(u[ok]).cuda(), temperature=t, **s)
            token, lp, kp = (x.cpu().numpy() for x in got)
            assert np.array_equal(token, want), (r, s, np.flatnonzero(token != want)[:5])
            x = (o.z[want] - o.z.max()) / np.longdouble(t)
            for y, total, off in ((lp, o.w.sum(), WEIGHT), (kp, o.value[ids].sum() / (ONE if o is cut else 1),
                                                            float(o.off[ids].sum() / o.value[ids].sum()))):
                ref = x - np.log(total)
                assert np.all(np.abs(y - ref) <= off + np.abs(ref) * (2.0 ** -24 * (1 + 1e-6)) + 1e-13), (r, s)
            tested += len(want)
    assert tested > 100 * rows
