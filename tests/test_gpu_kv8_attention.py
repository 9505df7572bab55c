"""Attention over the 8-bit cache against the float64 oracle: single rows and
runs, head groups, pages, lengths from none to thousands, split contexts, and
what must not reach a row."""
import numpy as np
import pytest
import torch

from kv8_helpers import BF16, F32, UNIT, Batch, attention_bound, dev, host, offsets, rounded
from oracle import kv8

pytestmark = pytest.mark.gpu


def _positions(new, lengths):
    return np.concatenate([np.arange(n - a, n) for a, n in zip(new, lengths)]).astype(int)


def _p_step(dtype, tiles):
    """Half a step of a probability as it enters the product: bf16 in runs of bf16 rows, 17 bits in single ones."""
    return 2.0 ** -24 if dtype is F32 else 2.0 ** -8 if tiles else 2.0 ** -16


def _check(b, q, new, out, dtype, scale, tiles):
    """Every output of a batch within its bound."""
    at, out = np.cumsum([0] + list(new)), host(out)
    for s, n in enumerate(b.lengths()):
        if not new[s]:
            continue
        pos = np.arange(n - new[s], n)
        ref, mass, reach = kv8.attend(q[at[s]:at[s + 1]], b.k[s].values(), b.v[s].values(), pos, scale)
        err = np.abs(out[at[s]:at[s + 1]] - ref)
        bound = attention_bound(ref, mass, reach, b.hd, n, scale, dtype, _p_step(dtype, tiles))
        assert np.all(err <= bound), (s, n, float((err - bound).max()), float((err / np.maximum(bound, 1e-30)).max()))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd,n_kv,rep", [(128, 2, 6), (128, 4, 7), (64, 12, 1), (64, 2, 8), (128, 1, 16), (64, 1, 17), (128, 1, 40)])
@pytest.mark.parametrize("page", [16, 64])
def test_single_rows(dtype, hd, n_kv, rep, page):
    """Lengths around every step of 16 and 32 tokens and beyond one workgroup round."""
    import paper_2606_02218_amd as rg
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 385, 1000]
    b = Batch(lens, n_kv, hd, page, seed=hd + rep)
    q = rounded(b.rng.normal(0, 1.5, (len(lens), n_kv * rep, hd)), dtype)
    args = (b.cache, dev(q, dtype), dev(b.tab), dev(b.lengths()))
    out = rg.kv8_attention(*args, max_len=1000)
    _check(b, q, [1] * len(lens), out, dtype, hd ** -0.5, False)
    # the same through offsets, another table order, a given output, no bound
    order = np.arange(len(lens))[::-1].copy()
    into = torch.full_like(out, 9.0)
    same = rg.kv8_attention(b.cache, args[1], dev(np.ascontiguousarray(b.tab[order])), args[3], offsets([1] * len(lens)),
                            tab_row=dev(order.astype(np.int32)), out=into, max_len=1000)
    assert same is into and torch.equal(into, out)
    _check(b, q, [1] * len(lens), rg.kv8_attention(*args), dtype, hd ** -0.5, False)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd,n_kv,rep", [(128, 2, 6), (128, 1, 7), (64, 3, 1), (64, 2, 8), (64, 1, 33), (128, 1, 128)])
@pytest.mark.parametrize("new,old", [([5, 1, 64], [0, 63, 64]), ([33, 0, 17, 40], [7, 9, 100, 200]), ([130], [0]),
                                     ([1, 2, 30], [600, 31, 0]), ([2, 3], [40, 5])])
def test_runs(dtype, hd, n_kv, rep, new, old):
    import paper_2606_02218_amd as rg
    b = Batch([a + o for a, o in zip(new, old)], n_kv, hd, 16, seed=hd + rep + len(new))
    rows = sum(new)
    q = rounded(b.rng.normal(0, 1.5, (rows, n_kv * rep, hd)), dtype)
    out = rg.kv8_attention(b.cache, dev(q, dtype), dev(b.tab), dev(b.lengths()), offsets(new))
    _check(b, q, new, out, dtype, hd ** -0.5, rows >= 4 * len(new))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [[1, 1], [3, 2], [9, 20]])
def test_split_contexts(dtype, new):
    """Few rows of long contexts are cut into chunks that a merge joins, in both passes; a bound below the longest
    sequence still computes it whole; the joined order is fixed."""
    import paper_2606_02218_amd as rg
    from paper_2606_02218_amd import _kv8
    b = Batch([5001, 1234], 2, 64, 16, seed=sum(new))
    q = rounded(b.rng.normal(0, 1.5, (sum(new), 8, 64)), dtype)
    off = None if new == [1, 1] else offsets(new)
    args = (b.cache, dev(q, dtype), dev(b.tab), dev(b.lengths()), off)
    lib = _kv8._library()
    tiles = sum(new) >= 8
    first = None
    for bound in (5001, 20000, 3000, 600, 1):
        need = lib.rg_kv8_attention_scratch(8, 2, 64, sum(new), 2, int(off is not None), bound)
        assert (need > 0) == (bound >= 3000)
        out = rg.kv8_attention(*args, max_len=bound)
        _check(b, q, new, out, dtype, 64 ** -0.5, tiles)
        again = rg.kv8_attention(*args, max_len=bound)
        assert torch.equal(out, again)
        first = out if first is None else first


def test_scale_and_peaked_scores():
    """A scale of the caller's; scores so far apart that most probabilities vanish, and the running maximum moves late."""
    import paper_2606_02218_amd as rg
    b = Batch([700, 300], 1, 64, 16, seed=2)
    for dtype in (BF16, F32):
        q = rounded(b.rng.normal(0, 1.0, (2, 4, 64)), dtype)
        q[:, 1] = rounded(q[:, 1] * 30, dtype)
        q[:, 2] = rounded(b.k[0].values()[650, 0] * 8, dtype)
        for scale in (0.05, 1.0, 3.0):
            out = rg.kv8_attention(b.cache, dev(q, dtype), dev(b.tab), dev(b.lengths()), scale=scale)
            _check(b, q, [1, 1], out, dtype, scale, False)
        run = rounded(b.rng.normal(0, 20.0, (12, 4, 64)), dtype)
        out = rg.kv8_attention(b.cache, dev(run, dtype), dev(b.tab), dev(b.lengths()), offsets([8, 4]))
        _check(b, run, [8, 4], out, dtype, 64 ** -0.5, True)


def test_queries_at_any_stride():
    import paper_2606_02218_amd as rg
    b = Batch([50, 90, 7], 2, 128, 16, seed=3)
    for dtype in (BF16, F32):
        base = dev(b.rng.normal(size=30 * 20 * 128 + 8).astype(np.float32), dtype)
        for new in ([1, 1, 1], [12, 14, 4]):
            n = sum(new)
            off = None if n == 3 else offsets(new)
            for q in (base[:n * 20 * 128].view(n, 20, 128)[:, 4:16], base[1:1 + n * 20 * 128].view(n, 20, 128)[:, 8:],
                      base[:20 * n * 128].view(20, n, 128).transpose(0, 1)[:, 2:14]):
                out = rg.kv8_attention(b.cache, q, dev(b.tab), dev(b.lengths()), off)
                assert torch.equal(out, rg.kv8_attention(b.cache, q.contiguous(), dev(b.tab), dev(b.lengths()), off))
                _check(b, host(q), new, out, dtype, 128 ** -0.5, n > 3)


def test_rows_that_see_nothing_and_rows_of_nobody():
    import paper_2606_02218_amd as rg
    b = Batch([3, 40, 0, 9], 2, 64, 16, seed=4)
    for dtype in (BF16, F32):
        # single rows: a padded batch with empty and negative lengths
        q = rounded(b.rng.normal(size=(4, 4, 64)), dtype)
        q[2] = np.nan                                       # a padding row's query is not read into anything
        length = np.array([3, 40, 0, -7], np.int32)
        out = rg.kv8_attention(b.cache, dev(q, dtype), dev(b.tab), dev(length), out=torch.full((4, 4, 64), 5.0, dtype=dtype, device="cuda"))
        assert torch.all(out[2:] == 0)
        _check(b, q, [1, 1, 0, 0], out, dtype, 0.125, False)
        long = rg.kv8_attention(b.cache, dev(q, dtype), dev(b.tab), dev(length), max_len=5000)
        assert torch.all(long[2:] == 0)
        # runs: sequence 0 has 3 tokens but 6 rows; the last rows belong to nobody
        new = [6, 7, 5, 4]
        q = rounded(b.rng.normal(size=(25, 4, 64)), dtype)
        q[:3] = np.nan
        length = np.array([3, 40, 0, 9], np.int32)
        for bound in (64, 5000):
            out = torch.full((25, 4, 64), 5.0, dtype=dtype, device="cuda")
            rg.kv8_attention(b.cache, dev(q, dtype), dev(b.tab), dev(length), offsets(new), out=out, max_len=bound)
            assert torch.all(out[:3] == 0) and torch.all(out[13:18] == 0) and torch.all(out[22:] == 5.0)
            seen = torch.cat([out[3:13], out[18:22]])
            _check(b, np.concatenate([q[3:13], q[18:22]]), [3, 7, 0, 4], seen, dtype, 0.125, True)
    z = torch.zeros(0, 4, 64, device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert rg.kv8_attention(b.cache, z, torch.zeros(0, 1, dtype=torch.int32, device="cuda"), none).shape == (0, 4, 64)


@pytest.mark.parametrize("hd", [64, 128])
def test_masked_tokens_do_not_touch_a_row(hd):
    """NaN codes behind the last token (every cache here starts full of them), and NaN keys and values at tokens that
    earlier rows of a run must not see; later rows get NaN in just the dims whose value is NaN, or whole for a key."""
    import paper_2606_02218_amd as rg
    for what in ("key", "value"):
        b = Batch([100, 70], 1, hd, 16, seed=hd)
        codes = (b.k if what == "key" else b.v)[0].codes
        codes[90, 0, 5] = 0x7F
        codes[75, 0, hd - 1] = 0xFF
        b.write()
        for dtype in (BF16, F32):
            for new in ([1, 1], [40, 3], [64, 64]):
                q = rounded(b.rng.normal(size=(sum(new), 3, hd)), dtype)
                out = host(rg.kv8_attention(b.cache, dev(q, dtype), dev(b.tab), dev(b.lengths()),
                                            None if new == [1, 1] else offsets(new)))
                pos = _positions(new, b.lengths())[:new[0]]
                nan = np.zeros((new[0], 3, hd), bool)
                if what == "key":
                    nan[pos >= 75] = True
                else:
                    nan[pos >= 90, :, 5] = True
                    nan[pos >= 75, :, hd - 1] = True
                assert np.array_equal(np.isnan(out[:new[0]]), nan), (what, dtype, new)
                assert np.all(np.isfinite(out[new[0]:]))


@pytest.mark.parametrize("hd,rep", [(64, 1), (64, 3), (128, 7)])
def test_nan_values_reach_just_the_rows_that_see_them(hd, rep):
    """One NaN value at a time, at places before, among and behind the rows of tiles: rows in sight get NaN in its dim."""
    import paper_2606_02218_amd as rg
    old, new = 30, 150
    q = None
    for at in (0, 29, 30, 31, 33, 47, 62, 63, 64, 70, 95, 96, 127, 128, 150, 178, 179):
        b = Batch([old + new], 1, hd, 16, seed=1)
        d = (7 * at) % hd
        b.v[0].codes[at, 0, d] = 0x7F
        b.write()
        q = rounded(b.rng.normal(size=(new, rep, hd)), BF16) if q is None else q
        nan = np.zeros((new, rep, hd), bool)
        nan[np.arange(old, old + new) >= at, :, d] = True
        for dtype in (BF16, F32):
            out = host(rg.kv8_attention(b.cache, dev(q, dtype), dev(b.tab), dev(b.lengths()), offsets([new])))
            assert np.array_equal(np.isnan(out), nan), (at, dtype)


def test_special_queries_stay_in_their_heads():
    import paper_2606_02218_amd as rg
    b = Batch([90, 33], 2, 64, 16, seed=6)
    for dtype in (BF16, F32):
        for new in ([1, 1], [20, 6]):
            n = sum(new)
            off = None if n == 2 else offsets(new)
            q = rounded(b.rng.normal(size=(n, 6, 64)), dtype)
            clean = rg.kv8_attention(b.cache, dev(q, dtype), dev(b.tab), dev(b.lengths()), off)
            q[0, 1, 3], q[n - 1, 4, 0], q[0, 5, 9] = np.nan, np.inf, -np.inf
            out = rg.kv8_attention(b.cache, dev(q, dtype), dev(b.tab), dev(b.lengths()), off)
            hit = torch.zeros(n, 6, dtype=torch.bool, device="cuda")
            hit[0, 1] = hit[n - 1, 4] = hit[0, 5] = True
            assert torch.all(out[hit].isnan()) and torch.equal(out[~hit], clean[~hit])


def test_lost_pages_make_their_rows_nan():
    """A page that is none of the pool's, or a length past the table: NaN for the rows that need it, in time that does
    not depend on the length, and the other rows as ever."""
    import paper_2606_02218_amd as rg
    b = Batch([100, 60, 50], 1, 64, 16, capacity=128, seed=7)
    for bad in (-1, b.pages, 2 ** 31 - 1, -2 ** 31):
        tab = b.tab.copy()
        tab[0, 4] = bad                                       # tokens 64 .. 79
        for new in ([1, 1, 1], [60, 9, 5]):
            n = sum(new)
            off = None if n == 3 else offsets(new)
            for bound in (128, 2000):
                q = dev(b.rng.normal(size=(n, 2, 64)).astype(np.float32), BF16)
                out = rg.kv8_attention(b.cache, q, dev(tab), dev(b.lengths()), off, max_len=bound)
                fine = rg.kv8_attention(b.cache, q, dev(b.tab), dev(b.lengths()), off, max_len=bound)
                lost = torch.zeros(n, dtype=torch.bool, device="cuda")
                lost[:new[0]] = torch.from_numpy(_positions(new, b.lengths())[:new[0]] >= 64).cuda()
                assert torch.all(out[lost].isnan()) and torch.equal(out[~lost], fine[~lost])
    q = dev(b.rng.normal(size=(3, 2, 64)).astype(np.float32), BF16)
    cap = b.width * 16
    out = rg.kv8_attention(b.cache, q, dev(b.tab), dev(np.array([cap + 1, 2 ** 31 - 1, 50], np.int32)))
    assert torch.all(out[:2].isnan()) and torch.all(out[2].isfinite())
    out = rg.kv8_attention(b.cache, q, dev(b.tab), dev(b.lengths()), tab_row=dev(np.array([3, -1, 2], np.int32)))
    assert torch.all(out[:2].isnan()) and torch.all(out[2].isfinite())
    q = dev(b.rng.normal(size=(30, 2, 64)).astype(np.float32), BF16)
    out = rg.kv8_attention(b.cache, q, dev(b.tab), dev(np.array([cap + 5, 2 ** 31 - 1, 50], np.int32)), offsets([10, 10, 10]))
    # rows of sequence 0 at positions cap - 5 .. cap + 4
    assert torch.all(out[5:20].isnan()) and torch.all(out[20:].isfinite())
    for off in ([0, 9, 3, 30], [-7, 0, 2, 100], [50, 60, 70, 80]):    # no access outside the buffers
        rg.kv8_attention(b.cache, q, dev(b.tab), dev(b.lengths()), dev(np.array(off, np.int32)))
    torch.cuda.synchronize()


def test_shared_pages_and_caches_past_32_bits():
    """Sequences that share a prefix's pages; pages whose bytes lie past 2^32 in the pool."""
    import paper_2606_02218_amd as rg
    b = Batch([64, 64, 64], 4, 128, 16, seed=8)
    b.tab[1:] = b.tab[0]
    q = rounded(b.rng.normal(size=(3, 8, 128)), BF16)
    out = rg.kv8_attention(b.cache, dev(q, BF16), dev(b.tab), dev(np.array([64, 33, 50], np.int32)))
    for r, n in enumerate((64, 33, 50)):
        ref, mass, reach = kv8.attend(q[r:r + 1], b.k[0].values(), b.v[0].values(), [n - 1], 128 ** -0.5)
        assert np.all(np.abs(host(out[r:r + 1]) - ref) <= attention_bound(ref, mass, reach, 128, n, 128 ** -0.5, BF16, 2.0 ** -16))
    pages = 700_000                                            # 4 heads x 2 KiB x 700000 = 5.7 GB
    big = rg.Kv8Cache.empty(pages, 4, 128, 16)
    far = np.arange(pages - 300, pages, 7)[:b.width * 3].reshape(3, -1)[:, :b.width].astype(np.int32)
    n = dev(np.array([64, 64, 64], np.int32))
    kv = dev(b.rng.normal(size=(3 * 64, 4, 128)).astype(np.float32), BF16)
    small = rg.Kv8Cache.empty(far.size, 4, 128, 16)
    near = np.arange(far.size, dtype=np.int32).reshape(far.shape)
    off = offsets([64, 64, 64])
    got = []
    for c, t in ((big, far), (small, near)):
        rg.kv8_append(c, kv, kv, dev(t), n, off)
        run = rg.kv8_attention(c, kv[:, :].repeat(1, 2, 1), dev(t), n, off)
        got.append((rg.kv8_attention(c, dev(q, BF16), dev(t), n), run))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_sequence_from_prompt_to_last_token(dtype):
    """The three operators as a decoder uses them: prompts in one ragged append, then single tokens with a chunk in
    between, each step's attention against the oracle's own cache of the same turned keys."""
    import paper_2606_02218_amd as rg
    n_kv, rep, hd, rot = 2, 3, 64, 48
    b = Batch([0, 0, 0], n_kv, hd, 32, capacity=150, seed=12)
    tab = dev(b.tab)
    cos, sin = rg.rope_table(150, rot, 1e4, scaling="bands", factor=4.0, length=64.0)
    ch, sh = host(cos), host(sin)
    for new in ([70, 33, 5], [1, 1, 1], [1, 1, 1], [17, 2, 6], [1, 1, 1], [0, 1, 40], [1, 1, 1]):
        old, rows = b.lengths(), sum(new)
        qkv = dev(b.rng.normal(size=(rows, (rep + 2) * n_kv, hd)).astype(np.float32), dtype)
        q, k, v = qkv[:, :rep * n_kv], qkv[:, rep * n_kv:-n_kv], qkv[:, -n_kv:]
        pos = np.concatenate([np.arange(o, o + a) for a, o in zip(new, old)]).astype(int)
        at = np.cumsum([0] + new)
        off = None if new == [1, 1, 1] else offsets(new)
        ln = dev((old + np.array(new)).astype(np.int32))
        turned = rg.kv8_append(b.cache, k, v, tab, ln, off, q=q, cos=cos, sin=sin)
        out = rg.kv8_attention(b.cache, turned, tab, ln, off)
        kt = kv8.rotate(host(k), ch[pos], sh[pos])
        for s in range(3):
            b.k[s].append(kt[at[s]:at[s + 1]])
            b.v[s].append(host(v)[at[s]:at[s + 1]])
        # a key within fp32 error of a rounding border may take the other code: one code step of that element.  The
        # oracle goes on with the codes the device holds, which the append's own tests check.
        got, want = b.snapshot(), b.image()
        assert np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2]) and np.array_equal(got[3], want[3])
        assert np.count_nonzero(got[0] != want[0]) <= 1e-4 * k.numel() + 1
        b2 = kv8._VALUES
        for s in range(3):
            n = len(b.k[s].codes)
            if n:
                held = b.logical(s, n, True) / np.repeat(b.k[s].scale, 16, 0)[:n, :, None]
                b.k[s].codes = kv8.e4m3_round(held)
                assert np.array_equal(b2[b.k[s].codes], held)
        _check(b, host(turned), new, out, dtype, hd ** -0.5, off is not None and rows >= 12)


def test_captured_and_replayed_with_eager_work_between():
    """Append and attention in one graph, split context and all, replayed on new inputs between eager calls on the same
    and on another cache; a second graph shares nothing with the first."""
    import paper_2606_02218_amd as rg
    caches = [Batch([900, 37, 0, 255], 2, 64, 16, capacity=1000, seed=20) for _ in range(2)]
    cos, sin = rg.rope_table(1000, 64)
    graphs = []
    for b in caches:
        st = dict(qkv=torch.zeros(4, 8, 64, dtype=BF16, device="cuda"), len=dev(b.lengths()), tab=dev(b.tab))

        def step(b=b, st=st):
            q = rg.kv8_append(b.cache, st["qkv"][:, 4:6], st["qkv"][:, 6:], st["tab"], st["len"], q=st["qkv"][:, :4], cos=cos, sin=sin)
            return rg.kv8_attention(b.cache, q, st["tab"], st["len"], max_len=1000)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        keep = [t.clone() for t in b.cache]
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        for t, k in zip(b.cache, keep):
            t.view(torch.uint8).copy_(k.view(torch.uint8))
        graphs.append((b, st, g, out, step))
    rng = np.random.default_rng(1)
    for i in range(6):
        for b, st, g, out, step in graphs:
            st["qkv"].copy_(dev(rng.normal(size=(4, 8, 64)).astype(np.float32), BF16))
            st["len"].add_(1)
        torch.cuda.synchronize()
        before = [[t.clone() for t in b.cache] for b, *_ in graphs]
        for b, st, g, out, step in graphs:
            g.replay()
        torch.cuda.synchronize()
        replayed = [(out.clone(), [t.clone() for t in b.cache]) for b, st, g, out, step in graphs]
        for (b, st, g, out, step), old, (want, cache) in zip(graphs, before, replayed):
            for t, k in zip(b.cache, old):
                t.view(torch.uint8).copy_(k.view(torch.uint8))
            eager = step()
            assert torch.equal(eager, want)
            for t, k in zip(b.cache, cache):
                assert torch.equal(t.view(torch.uint8), k.view(torch.uint8))


def test_calls_on_two_streams_at_once():
    """Two batches of split contexts on two streams, in flight together: each call's scratch is its own."""
    import paper_2606_02218_amd as rg
    bs = [Batch([3000 + 100 * i, 777], 2, 64, 16, seed=30 + i) for i in range(2)]
    qs = [dev(b.rng.normal(size=(2, 8, 64)).astype(np.float32), BF16) for b in bs]
    rest = [(dev(b.tab), dev(b.lengths())) for b in bs]
    want = [rg.kv8_attention(b.cache, q, *r, max_len=3200) for b, q, r in zip(bs, qs, rest)]
    streams = [torch.cuda.Stream() for _ in bs]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(20):
        for i in range(2):
            outs[i].append(rg.kv8_attention(bs[i].cache, qs[i], *rest[i], max_len=3200, stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in outs[i])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd,n,dead", [(64, 200, 70), (128, 200, 33), (128, 3000, 2100), (64, 2500, 1), (64, 90, 90)])
def test_scores_past_the_range(dtype, hd, n, dead):
    """Scores that overflow to -inf have no weight, whichever steps, waves and chunks they fill; a row with no others
    is NaN, as a softmax over nothing."""
    import paper_2606_02218_amd as rg
    b = Batch([0], 2, hd, 16, capacity=n, seed=40)
    k = rounded(b.rng.normal(size=(n, 2, hd)), BF16)
    k[:, :, 0] = np.where(np.arange(n) < dead, 100.0, 0.0)[:, None]
    b.k[0].append(k)
    b.v[0].append(rounded(b.rng.normal(size=(n, 2, hd)), BF16))
    b.write()
    keys, values = b.k[0].values(), b.v[0].values()
    assert np.all(keys[:dead, :, 0] > 90) and np.all(keys[dead:, :, 0] == 0)
    for new in (1, 30):
        q = rounded(b.rng.normal(size=(new, 6, hd)), dtype)
        q[:, :, 0] = rounded(np.full((new, 6), -3e37), dtype)         # -3e37 * 90 < -3.4e38
        out = host(rg.kv8_attention(b.cache, dev(q, dtype), dev(b.tab), dev(b.lengths()), offsets([new]), max_len=n))
        pos = np.arange(n - new, n) - dead
        lost = pos < 0
        assert np.all(np.isnan(out[lost]))
        if not lost.all():
            ref, mass, reach = kv8.attend(q[~lost], keys[dead:], values[dead:], pos[~lost], hd ** -0.5)
            bound = attention_bound(ref, mass, reach, hd, n, hd ** -0.5, dtype, _p_step(dtype, new > 3))
            assert np.all(np.abs(out[~lost] - ref) <= bound)


def test_lengths_below_zero_hold_nothing():
    """As a length of zero, in single rows and runs, to the smallest integer."""
    import paper_2606_02218_amd as rg
    b = Batch([40, 60, 50], 2, 64, 16, seed=41)
    for dtype in (BF16, F32):
        for new in ([1, 1, 1], [20, 9, 5]):
            n = sum(new)
            off = None if n == 3 else offsets(new)
            x = dev(rounded(b.rng.normal(size=(n, 4, 64)), dtype), dtype)
            rows = slice(new[0], new[0] + new[1])
            want = rg.kv8_attention(b.cache, x, dev(b.tab), dev(b.lengths()), off)
            want[rows] = 0
            for low in (0, -1, -7, -2 ** 31 + 3, -2 ** 31):
                ln = dev(np.array([40, low, 50], np.int32))
                assert torch.equal(rg.kv8_attention(b.cache, x, dev(b.tab), ln, off), want), low
                before = b.snapshot()
                rg.kv8_append(b.cache, x[:, :2], x[:, 2:], dev(b.tab), dev(np.full(3, low, np.int32)), off)
                assert all(np.array_equal(a, c) for a, c in zip(b.snapshot(), before)), low


@pytest.mark.parametrize("page", [256, 1024])
@pytest.mark.parametrize("new", [1, 50])
def test_large_pages(page, new):
    """Pages of many blocks, lengths that end inside one and at its end; sizes given as other integers."""
    import paper_2606_02218_amd as rg
    for n in (page - 1, page, page + 1, 2 * page):
        b = Batch([n, 70], 2, 64, page, capacity=2 * page, seed=42)
        q = rounded(b.rng.normal(size=(2 * new, 8, 64)), BF16)
        out = rg.kv8_attention(b.cache, dev(q, BF16), dev(b.tab), dev(b.lengths()), offsets([new, new]),
                               max_len=np.int64(2 * page))
        _check(b, q, [new, new], out, BF16, 64 ** -0.5, new > 3)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_captured_runs(dtype):
    """A prompt's piece appended and attended to in a graph, contexts in chunks, replayed with eager work between."""
    import paper_2606_02218_amd as rg
    b = Batch([1500, 200], 2, 128, 16, capacity=1700, seed=43)
    assert rg.load_library().rg_kv8_attention_scratch(8, 2, 128, 60, 2, 1, 1700) > 0
    x = torch.zeros(60, 12, 128, dtype=dtype, device="cuda")
    tab, off, ln = dev(b.tab), offsets([40, 20]), dev(b.lengths())
    cos, sin = rg.rope_table(1700, 128)

    def step():
        q = rg.kv8_append(b.cache, x[:, 8:10], x[:, 10:], tab, ln, off, q=x[:, :8], cos=cos, sin=sin)
        return rg.kv8_attention(b.cache, q, tab, ln, off, max_len=1700)

    def put(to):
        for t, k in zip(b.cache, to):
            t.view(torch.uint8).copy_(k.view(torch.uint8))

    keep = [t.clone() for t in b.cache]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for i in range(4):
        put(keep)
        x.copy_(dev(b.rng.normal(size=(60, 12, 128)).astype(np.float32), dtype))
        ln.copy_(dev(b.lengths() + 5 * i))
        want = step().clone()
        cache = [t.clone() for t in b.cache]
        torch.cuda.synchronize()
        put(keep)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.all(out.isfinite())
        for t, k in zip(b.cache, cache):
            assert torch.equal(t.view(torch.uint8), k.view(torch.uint8))


def test_a_whole_step_on_a_given_stream():
    """rope_table, append and attention on a stream of the caller's, the results used there."""
    import paper_2606_02218_amd as rg
    b = Batch([2500, 30], 2, 64, 16, capacity=2600, seed=44)
    x = dev(b.rng.normal(size=(2, 12, 64)).astype(np.float32), BF16)
    ln = dev(b.lengths() + 1)
    keep = [t.clone() for t in b.cache]
    tab, got = dev(b.tab), []
    for stream in (None, torch.cuda.Stream()):
        for t, k in zip(b.cache, keep):
            t.view(torch.uint8).copy_(k.view(torch.uint8))
        torch.cuda.synchronize()
        cos, sin = rg.rope_table(2600, 64, stream=stream)
        q = rg.kv8_append(b.cache, x[:, 8:10], x[:, 10:], tab, ln, q=x[:, :8], cos=cos, sin=sin, stream=stream)
        got.append(rg.kv8_attention(b.cache, q, tab, ln, max_len=2600, stream=stream))
        torch.cuda.synchronize()
    assert torch.equal(*got)


@pytest.mark.parametrize("dtype,n_kv,rep,hd", [(BF16, 12, 1, 64), (F32, 5, 2, 64), (BF16, 2, 6, 128), (BF16, 1, 40, 64)])
@pytest.mark.parametrize("rows", [64, 65, 131, 700])
def test_many_ragged_rows(dtype, n_kv, rep, hd, rows):
    """Rows enough to be taken by length: each gets what it gets in a small batch, whatever the lengths (none, equal
    ones, past the bound given and past the table)."""
    import paper_2606_02218_amd as rg
    b = Batch([300, 270], n_kv, hd, 16, capacity=304, seed=50)
    rng = np.random.default_rng(rows)
    q = dev(rng.normal(size=(rows, n_kv * rep, hd)).astype(np.float32), dtype)
    tab = dev(b.tab[rng.integers(0, 2, size=rows)])
    some = -(-257 // (n_kv * -(-rep // 16)))                      # the fewest rows that take four waves
    for ln in (rng.integers(1, 271, size=rows), np.full(rows, 77), np.repeat([0, 1, 270], rows)[::3][:rows],
               np.where(rng.random(rows) < 0.1, rng.choice([2 ** 31 - 1, 400, -3], size=rows), rng.integers(0, 271, size=rows))):
        ln = dev(ln.astype(np.int32))
        for bound in (270, 40):
            out = rg.kv8_attention(b.cache, q, tab, ln, max_len=bound)
            few = min(some, 63)
            for a in range(0, rows, few):
                a = max(min(a, rows - few), 0)
                part = rg.kv8_attention(b.cache, q[a:a + few], tab[a:a + few], ln[a:a + few], max_len=bound)
                got = out[a:a + few]
                if few * n_kv * -(-rep // 16) > 256:
                    assert torch.equal(got.isnan(), part.isnan()) and torch.equal(got.nan_to_num(7), part.nan_to_num(7))
                else:                                             # eight waves: other sums
                    assert torch.allclose(got.float(), part.float(), rtol=2 * UNIT[dtype] + 2 ** -16, atol=2 ** -16, equal_nan=True)


@pytest.mark.parametrize("n_kv,rep", [(2, 6), (1, 64)])
def test_many_sequences_of_runs(n_kv, rep):
    """More sequences than a wave has lanes, some without rows: each run gets what it gets in a small batch."""
    import paper_2606_02218_amd as rg
    b = Batch([300, 270], n_kv, 64, 16, capacity=304, seed=51)
    rng = np.random.default_rng(3)
    for seqs in (64, 65, 200):
        new = rng.choice([0, 3, 17, 40], size=seqs)
        new[:2] = 0, 60
        ln = np.maximum(rng.integers(0, 271, size=seqs), new // 2)        # the first rows of some are padding
        tab = b.tab[rng.integers(0, 2, size=seqs)]
        off = np.concatenate([[0], np.cumsum(new)])
        rows = int(off[-1])
        assert rows >= 4 * seqs
        q = dev(rng.normal(size=(rows, n_kv * rep, 64)).astype(np.float32), BF16)
        out = rg.kv8_attention(b.cache, q, dev(tab), dev(ln.astype(np.int32)), dev(off.astype(np.int32)), max_len=270)
        for a in range(0, seqs, 10):
            z = min(a + 10, seqs)
            r = slice(int(off[a]), int(off[z]))
            if off[z] - off[a] < 4 * (z - a):
                continue
            part = rg.kv8_attention(b.cache, q[r], dev(tab[a:z]), dev(ln[a:z].astype(np.int32)),
                                    dev((off[a:z + 1] - off[a]).astype(np.int32)), max_len=270)
            assert torch.equal(out[r], part)


def test_calls_without_rows():
    """No rows, with and without sequences, leave nothing to do; sequences without rows do not disturb the others."""
    import paper_2606_02218_amd as rg
    b = Batch([40, 60], 2, 64, 16, seed=52)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    for dtype in (BF16, F32):
        q = torch.zeros(0, 4, 64, dtype=dtype, device="cuda")
        assert rg.kv8_attention(b.cache, q, dev(b.tab)[:0], none).shape == (0, 4, 64)
        assert rg.kv8_attention(b.cache, q, dev(b.tab), dev(b.lengths()), offsets([0, 0]), max_len=4000).shape == (0, 4, 64)
        cos, sin = rg.rope_table(4, 64)
        assert rg.rope(q, none, cos, sin).shape == (0, 4, 64)
        assert rg.rope(torch.zeros(3, 0, 64, dtype=dtype, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"), cos,
                       sin).shape == (3, 0, 64)
        x = rounded(b.rng.normal(size=(9, 4, 64)), dtype)
        out = rg.kv8_attention(b.cache, dev(x, dtype), dev(b.tab), dev(b.lengths()), offsets([0, 9]))
        _check(b, x, [0, 9], out, dtype, 64 ** -0.5, True)
    torch.cuda.synchronize()
