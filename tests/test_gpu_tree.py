"""Drafted trees over the 8-bit cache against the float64 oracle: masks and
positions, attention of the nodes, the accepted path's move, and a round of them
together."""
import ctypes

import numpy as np
import pytest
import torch

from kv8_helpers import BF16, F32, Batch, attention_bound, dev, host, offsets, rounded
from oracle import kv8, tree

pytestmark = pytest.mark.gpu


def parents(n, kind, rng):
    if kind == "chain":
        return np.arange(n) - 1
    if kind == "star":
        return np.minimum(np.arange(n) - 1, 0)
    if kind == "forest":
        return np.array([-1 if rng.random() < 0.3 else int(rng.integers(-1, i)) for i in range(n)], int)
    return np.array([-1] + [int(rng.integers(max(0, i - 5), i)) for i in range(1, n)], int)


def words_of(nodes):
    return max(1, -(-max(nodes) // 64))


def as_mask(m):
    return dev(m.view(np.int64))


def all_masks(trees, words, ctx, lens):
    got = [tree.masks(p, words, c, max(len(p) - n, 0)) for p, c, n in zip(trees, ctx, lens)]
    return np.concatenate([m for m, _ in got]), np.concatenate([p for _, p in got])


# ---------------------------------------------------------------- masks
@pytest.mark.parametrize("kind", ["chain", "star", "forest", "tree"])
@pytest.mark.parametrize("nodes,words", [([1], 1), ([5, 0, 64, 1, 63], 1), ([65, 128, 3], 2), ([200, 31, 129], 4), ([300], 64),
                                         ([130, 70], 1), ([2500, 40], 40), ([0, 0, 7], 3)])
def test_masks(kind, nodes, words):
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(len(nodes) + words)
    trees = [parents(n, kind, rng) if n else np.zeros(0, int) for n in nodes]
    ctx = rng.integers(0, 5000, len(nodes))
    lens = ctx + np.array(nodes)
    mask, pos = rg.kv8_tree(dev(np.concatenate(trees).astype(np.int32)), dev(lens.astype(np.int32)), offsets(nodes), words=words)
    want, at = all_masks(trees, words, ctx, lens)
    assert mask.dtype == torch.int64 and mask.shape == (sum(nodes), words)
    assert np.array_equal(mask.cpu().numpy().view(np.uint64), want)
    assert np.array_equal(pos.cpu().numpy(), at)


def test_masks_of_wrong_parents_and_padding():
    """Parents that are none, nodes behind them, sequences with fewer tokens than rows, rows of nobody."""
    import paper_2606_02218_amd as rg
    trees = [np.array([-1, 5, 1, 0, -2, 4, 6]), np.array([-1, 0, 1, 2, 1]), np.array([0, -1]), np.array([-1, 0, 1])]
    nodes, lens = [len(t) for t in trees], [17, 3, 2, 0]
    parent = np.concatenate(trees + [np.array([-1, 0, 1])]).astype(np.int32)     # three rows of nobody
    off = offsets(nodes)
    lib = rg.load_library()
    mask = torch.full((len(parent), 2), 77, dtype=torch.int64, device="cuda")
    pos = torch.full((len(parent),), 77, dtype=torch.int32, device="cuda")
    p, n = dev(parent), dev(np.array(lens, np.int32))
    rg.kv8_tree(p, n, off, words=2)                                              # sets the argument types up
    assert lib.rg_kv8_tree(p.data_ptr(), off.data_ptr(), n.data_ptr(), 4, len(parent), 2, mask.data_ptr(), pos.data_ptr(),
                           torch.cuda.current_stream().cuda_stream) == 0
    want, at = all_masks(trees, 2, [max(a - b, 0) for a, b in zip(lens, nodes)], lens)
    assert np.array_equal(mask.cpu().numpy().view(np.uint64)[:-3], want) and np.array_equal(pos.cpu().numpy()[:-3], at)
    assert bool((mask[-3:] == 77).all()) and bool((pos[-3:] == 77).all())


def long_masks(parent, words, context, first=0):
    """tree.masks for trees whose paths are too long to be written out: by each node's parent."""
    mask, pos = np.zeros((len(parent), words), np.uint64), np.full(len(parent), -1)
    for i in range(first, len(parent)):
        p = int(parent[i])
        if not -1 <= p < i or (p >= first and pos[p] < 0):
            continue
        pos[i] = context
        if p >= first:
            mask[i], pos[i] = mask[p], pos[p] + 1
        if i < 64 * words:
            mask[i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
    return mask, pos


@pytest.mark.parametrize("kind", ["chain", "star", "forest", "tree", "wrong"])
@pytest.mark.parametrize("n,words", [(2048, 64), (2049, 33), (4096, 64), (4100, 64), (70001, 7), (300000, 1)])
def test_masks_of_long_trees(kind, n, words):
    """Work grows with the nodes, not with their square: a chain of 300 thousand, wrong parents, padding and short
    trees beside them."""
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(n)
    p = parents(n, "tree" if kind == "wrong" else kind, rng)
    if kind == "wrong":                                # what is behind these is nothing
        at = rng.choice(n, 5, replace=False)
        p[at] = [-2, -2 ** 31, 2 ** 31 - 1, at[3], min(at[4] + 70, n)]
        p[rng.choice(n, n // 30, replace=False)] = -1
        p[n - 40] = 2
    side = parents(65, "tree", rng)
    first = 77 if kind == "forest" else 0              # rows that are padding
    lens = [9 + 65, n - first if first else n + 1234, 5 + 65]
    parent = np.concatenate([side, p, side]).astype(np.int32)
    mask, pos = rg.kv8_tree(dev(parent), dev(np.array(lens, np.int32)), offsets([65, n, 65]), words=words)
    want = [long_masks(side, words, 9), long_masks(p, words, 0 if first else 1234, first), long_masks(side, words, 5)]
    if n < 2100:
        assert all(np.array_equal(a, b) for a, b in zip(want[1], tree.masks(p, words, 0 if first else 1234, first)))
    assert np.array_equal(pos.cpu().numpy(), np.concatenate([x[1] for x in want]))
    assert np.array_equal(mask.cpu().numpy().view(np.uint64), np.concatenate([x[0] for x in want]))


# ---------------------------------------------------------------- attention
P_STEP = {BF16: 2.0 ** -8, F32: 2.0 ** -24}      # half a step of a probability as it enters the product


def check(b, q, nodes, mask, out, dtype, scale=None, skip=()):
    at, out = np.cumsum([0] + list(nodes)), host(out)
    scale = b.hd ** -0.5 if scale is None else scale
    for s, n in enumerate(b.lengths()):
        r = slice(at[s], at[s + 1])
        if not nodes[s] or s in skip:
            continue
        sees = tree.seen(mask[r], n, nodes[s])
        ref, mass, reach = tree.attend(q[r], b.k[s].values(), b.v[s].values(), sees, scale)
        err = np.abs(out[r] - ref)
        bound = attention_bound(ref, mass, reach, b.hd, n, scale, dtype, P_STEP[dtype])
        assert np.all(err <= bound), (s, n, nodes[s], float((err - bound).max()))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd,n_kv,rep", [(128, 2, 6), (128, 1, 7), (64, 3, 1), (64, 2, 8), (64, 1, 33), (128, 1, 128)])
@pytest.mark.parametrize("nodes,old", [([1], [0]), ([5, 1, 9], [0, 63, 64]), ([33, 0, 17, 40], [7, 9, 100, 200]),
                                       ([64, 70, 130], [31, 0, 300]), ([3, 2], [600, 31])])
def test_attention(dtype, hd, n_kv, rep, nodes, old):
    import paper_2606_02218_amd as rg
    b = Batch([a + c for a, c in zip(nodes, old)], n_kv, hd, 16 if rep % 2 else 64, seed=hd + rep + len(nodes))
    trees = [parents(n, "tree", b.rng) if n else np.zeros(0, int) for n in nodes]
    mask, _ = all_masks(trees, words_of(nodes), old, b.lengths())
    q = rounded(b.rng.normal(0, 1.5, (sum(nodes), n_kv * rep, hd)), dtype)
    args = (b.cache, dev(q, dtype), dev(b.tab), dev(b.lengths()), offsets(nodes), as_mask(mask))
    out = rg.kv8_tree_attention(*args, max_len=int(b.lengths().max()))
    assert out.dtype == dtype and out.shape == q.shape
    check(b, q, nodes, mask, out, dtype)
    # strided queries, another table order, a given output, no bound
    order = np.arange(len(nodes))[::-1].copy()
    wide = torch.zeros(sum(nodes), n_kv * rep + 3, hd + 5, device="cuda", dtype=dtype)
    wide[:, 1:-2, 3:-2] = args[1]
    into = torch.full_like(out, 9.0)
    same = rg.kv8_tree_attention(b.cache, wide[:, 1:-2, 3:-2], dev(np.ascontiguousarray(b.tab[order])), *args[3:],
                                 tab_row=dev(order.astype(np.int32)), out=into, scale=0.05)
    assert same is into
    check(b, q, nodes, mask, same, dtype, 0.05)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("nodes,old", [([17, 64], [5000, 37]), ([3], [9001]), ([90, 1, 0, 30], [2050, 6000, 100, 0])])
def test_split_contexts(dtype, nodes, old):
    """Contexts cut into chunks, a bound that is too small among them, and the join."""
    import paper_2606_02218_amd as rg
    b = Batch([a + c for a, c in zip(nodes, old)], 1, 128, 64, seed=sum(nodes))
    trees = [parents(n, "forest", b.rng) if n else np.zeros(0, int) for n in nodes]
    mask, _ = all_masks(trees, words_of(nodes), old, b.lengths())
    q = rounded(b.rng.normal(0, 1.5, (sum(nodes), 6, 128)), dtype)
    args = (b.cache, dev(q, dtype), dev(b.tab), dev(b.lengths()), offsets(nodes), as_mask(mask))
    for bound in (int(b.lengths().max()), 1500, None):
        check(b, q, nodes, mask, rg.kv8_tree_attention(*args, max_len=bound), dtype)
    again = [rg.kv8_tree_attention(*args) for _ in range(3)]
    assert all(torch.equal(again[0], x) for x in again)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd,seqs,most", [(128, 40, 60), (64, 64, 60), (64, 65, 60), (128, 64, 15), (64, 65, 15), (128, 200, 10)])
def test_more_than_a_round_of_workgroups(dtype, hd, seqs, most):
    """Up to 64 sequences the longest go first, equal lengths and empty ones among them; past 64 in their order."""
    import paper_2606_02218_amd as rg
    rng = np.random.default_rng(seqs)
    nodes = [int(n) for n in rng.integers(0, most, seqs)]
    old = [int(n) for n in rng.choice([0, 5, 130, 130, 301], seqs)]
    b = Batch([a + c for a, c in zip(nodes, old)], 2, hd, 32, seed=seqs)
    trees = [parents(n, "tree", b.rng) if n else np.zeros(0, int) for n in nodes]
    mask, _ = all_masks(trees, 1, old, b.lengths())
    assert (sum(nodes) * 6 // 16 + seqs) * 2 > 256
    q = rounded(b.rng.normal(0, 1.5, (sum(nodes), 12, hd)), dtype)
    out = rg.kv8_tree_attention(b.cache, dev(q, dtype), dev(b.tab), dev(b.lengths()), offsets(nodes), as_mask(mask), max_len=400)
    check(b, q, nodes, mask, out, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_any_mask(dtype):
    """Masks that are no tree's: random bits, without the node itself, empty ones, bits past the nodes."""
    import paper_2606_02218_amd as rg
    nodes, old = [40, 9, 130, 5], [0, 0, 20, 3]
    b = Batch([a + c for a, c in zip(nodes, old)], 2, 64, 32, seed=5)
    mask = b.rng.integers(0, 2 ** 63, (sum(nodes), 3)).astype(np.uint64) * np.uint64(2) + np.uint64(1)
    mask[::5] = 0                                       # with no context these rows see nothing
    mask[1::7] = np.uint64(2 ** 64 - 1)
    q = rounded(b.rng.normal(0, 1.5, (sum(nodes), 4, 64)), dtype)
    out = rg.kv8_tree_attention(b.cache, dev(q, dtype), dev(b.tab), dev(b.lengths()), offsets(nodes), as_mask(mask))
    check(b, q, nodes, mask, out, dtype)
    empty = [i for i in range(0, 49) if i % 5 == 0 and i % 7 != 1]
    assert not host(out)[empty].any()
    # one word of the three: nodes past it have no bit
    one = rg.kv8_tree_attention(b.cache, dev(q, dtype), dev(b.tab), dev(b.lengths()), offsets(nodes), as_mask(mask[:, :1].copy()))
    check(b, q, nodes, mask[:, :1], one, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_padding_and_rows_of_nobody(dtype):
    """Sequences with fewer tokens than rows, of length 0 and below; rows behind the last sequence stay as they were."""
    import paper_2606_02218_amd as rg
    nodes, lens = [6, 4, 5], [3, 0, 40]
    b = Batch(lens, 2, 128, 16, seed=3)
    rows = sum(nodes) + 4
    mask = np.full((rows, 1), 2 ** 64 - 1, np.uint64)
    q = rounded(b.rng.normal(0, 1.5, (rows, 6, 128)), dtype)
    for cut in (0, -7):
        n = b.lengths()
        n[1] = cut
        out = torch.full((rows, 6, 128), 9.0, device="cuda", dtype=dtype)
        rg.kv8_tree_attention(b.cache, dev(q, dtype), dev(b.tab), dev(n), offsets(nodes), as_mask(mask), out=out)
        check(b, q, nodes, mask, out, dtype)
        assert not host(out)[:3].any() and not host(out)[6:10].any() and (host(out)[-4:] == 9.0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("split", [False, True])
def test_what_a_node_does_not_see(dtype, split):
    """NaN codes in nodes: those that see them are NaN in the dims that hold them, the others exact.  NaN keys likewise."""
    import paper_2606_02218_amd as rg
    old = 3000 if split else 45
    n, hd = 40, 64
    b = Batch([old + n], 1, hd, 16, seed=8)
    p = parents(n, "tree", b.rng)
    mask, _ = tree.masks(p, 1, old)
    q = rounded(b.rng.normal(0, 1.5, (n, 2, hd)), dtype)
    args = (dev(q, dtype), dev(b.tab), dev(b.lengths()), offsets([n]), as_mask(mask))
    clean = host(rg.kv8_tree_attention(b.cache, *args))
    bad_v, bad_k = 11, 7
    page, sub = b.places(0, -(-(old + n) // 16))
    v, k = b.cache.v.view(torch.uint8), b.cache.k.view(torch.uint8)
    t = old + bad_v
    for d in (5, 33):
        v[int(page[t // 16]), 0, int(sub[t // 16]), (t % 16 // 4) * 4 * hd + d * 4 + t % 4] = 0x7F
    out = host(rg.kv8_tree_attention(b.cache, *args))
    sees = tree.seen(mask, old + n, n)
    for i in range(n):
        if sees[i, t]:
            assert np.isnan(out[i][:, [5, 33]]).all()
            rest = [d for d in range(hd) if d not in (5, 33)]
            assert np.array_equal(out[i][:, rest], clean[i][:, rest])
        else:
            assert np.array_equal(out[i], clean[i]), i
    t = old + bad_k
    k[int(page[t // 16]), 0, int(sub[t // 16]), (9 // 16) * 256 + (t % 16) * 16 + 9] = 0xFF
    out2 = host(rg.kv8_tree_attention(b.cache, *args))
    for i in range(n):
        if sees[i, t]:
            assert np.isnan(out2[i]).all()
        else:
            assert np.array_equal(out2[i], out[i], equal_nan=True), i


def cuts(b, n_q, nodes, words, bound, dtype):
    """Whether the call takes 32 columns a workgroup, and in how many chunks, by the rule that the library states
    beside its plan; the chunks are those that its scratch has room for."""
    import paper_2606_02218_amd as rg
    rep, rows, seqs = n_q // b.n_kv, sum(nodes), len(nodes)
    of = lambda cols: (rows * rep // cols + seqs // 2 + 1) * b.n_kv  # noqa: E731
    cut = 1 if bound < 2048 else max(1, min((768 if dtype == BF16 else 512) // of(32), bound // 640))
    wide = rows * rep // seqs >= 64 and of(32) * cut >= 384
    want = cut if wide else 1 if bound < 2048 else max(1, min(256 // of(16), bound // 640))
    lib = rg.load_library()
    lib.rg_kv8_tree_attention_scratch.restype = ctypes.c_int64
    size = lib.rg_kv8_tree_attention_scratch(int(dtype == BF16), n_q, b.n_kv, b.hd, rows, seqs, words, bound)
    n = size // (4 * rows * n_q * (b.hd + 2)) or 1
    chunk = -(-(-(-bound // min(want, 64))) // 64) * 64
    assert n == -(-bound // chunk), (n, want, chunk)
    return wide, n


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n_kv,rep,n,wide,old,bound,chunks", [
    (1, 2, 40, False, 45, 85, 1), (1, 2, 40, False, 64, 104, 1), (1, 2, 40, False, 20, 60, 1), (2, 70, 33, False, 1993, 2026, 1),
    (1, 2, 40, False, 3000, 3040, 4), (1, 2, 40, False, 45, 1 << 14, 25), (24, 11, 70, True, 45, 115, 1),
    (24, 11, 70, True, 20, 90, 1), (24, 11, 70, True, 3000, 3070, 1), (8, 11, 70, True, 3000, 3070, 2)])
def test_nan_values_of_the_context(n_kv, rep, n, wide, old, bound, chunks, hd, dtype):
    """Every node sees the context: a NaN value there makes a dim of all of them NaN, in the step that also holds the
    first nodes as in those before it, and nothing else."""
    import paper_2606_02218_amd as rg
    b = Batch([old + n], n_kv, hd, 16, seed=old + hd)
    mask, _ = tree.masks(parents(n, "tree", b.rng), 2, old)
    mask[n // 2] = 0                                    # sees the context alone
    is_wide, pieces = cuts(b, n_kv * rep, [n], 2, bound, dtype)
    assert is_wide == wide and min(pieces, 2) == min(chunks, 2)
    q = rounded(b.rng.normal(0, 1.5, (n, n_kv * rep, hd)), dtype)
    args = (b.cache, dev(q, dtype), dev(b.tab), dev(b.lengths()), offsets([n]), as_mask(mask))
    clean = host(rg.kv8_tree_attention(*args, max_len=bound))
    page, sub = b.places(0, -(-(old + n) // 16))
    v = b.cache.v.view(torch.uint8)
    last = n_kv - 1
    for t in sorted({0, 7, old // 32 * 32 - 1, old // 32 * 32, old - 1} - {-1, old}):
        d = (5 * t + 3) % hd
        at = int(page[t // 16]), last, int(sub[t // 16]), (t % 16 // 4) * 4 * hd + d * 4 + t % 4
        was = v[at].item()
        v[at] = 0x7F if t % 2 else 0xFF
        out = host(rg.kv8_tree_attention(*args, max_len=bound))
        assert np.isnan(out[:, last * rep:, d]).all(), t
        out[:, last * rep:, d] = clean[:, last * rep:, d]
        assert np.array_equal(out, clean), t
        v[at] = was


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n_kv,rep,n,wide,bound", [(1, 2, 40, False, 900), (1, 2, 40, False, 3100), (24, 11, 70, True, 900),
                                                   (3, 11, 70, True, 3100)])
def test_scores_of_minus_infinity(n_kv, rep, n, wide, bound, hd, dtype):
    """A row that sees tokens, none of them with a weight, is NaN as in kv8_attention; one that sees nothing is zero;
    one token with a weight is enough, whatever the chunks."""
    import paper_2606_02218_amd as rg
    old, nodes = [45, 0, 3000 if bound > 2048 else 300], [n, n, n]
    b = Batch([c + n for c in old], n_kv, hd, 16, seed=n)
    mask = np.concatenate([tree.masks(parents(n, "tree", b.rng), 2, c)[0] for c in old])
    mask[n + 3] = mask[n + 17] = 0                       # with no context these rows see nothing
    is_wide, pieces = cuts(b, n_kv * rep, nodes, 2, bound, dtype)
    assert is_wide == wide and (pieces > 1) == (bound > 2048)
    b.cache.k.view(torch.uint8).fill_(0x40)              # 2
    b.cache.k_scale.fill_(1.0)
    q = np.zeros((3 * n, n_kv * rep, hd))
    q[:, :, 0] = -3.0e38
    q[:, 1::2, 0] = 0.0                                  # every other head's scores are 0
    args = (b.cache, dev(q, dtype), dev(b.tab), dev(b.lengths()), offsets(nodes), as_mask(mask))
    out = host(rg.kv8_tree_attention(*args, max_len=bound))
    none = [n + 3, n + 17]
    some = [i for i in range(3 * n) if i not in none]
    assert not out[none].any() and np.isnan(out[some][:, ::2]).all() and np.isfinite(out[some][:, 1::2]).all()
    one = rg.kv8_attention(b.cache, args[1][:3], args[2], args[3])
    assert np.isnan(host(one)[:, ::2]).all()
    page, sub = b.places(2, 1)
    k = b.cache.k.view(torch.uint8)
    k[int(page[0]), :, int(sub[0])] = 0                  # 16 tokens of the third sequence have scores of 0
    out = host(rg.kv8_tree_attention(*args, max_len=bound))
    mean = b.v[2].values()[:16].mean(0).repeat(rep, 0)
    # 16 exact probabilities of 1/16, sums of 16 terms, one rounding of the output
    bound_ = np.abs(b.v[2].values()[:16]).mean(0).repeat(rep, 0) * 16 * 2.0 ** -24 + np.abs(mean) * 1.01 * P_STEP[dtype] + 1e-30
    assert np.all(np.abs(out[2 * n:, ::2] - mean[::2]) <= bound_[::2])
    assert np.isnan(out[:n, ::2]).all() and not out[none].any()


def test_lost_pages():
    """Pages outside the pool or the table: NaN where a row sees a token of theirs, nothing elsewhere."""
    import paper_2606_02218_amd as rg
    nodes, old = [30, 30, 30], [40, 40, 40]
    b = Batch([70, 70, 70], 2, 64, 16, capacity=96, seed=4)
    p = [parents(30, "star", b.rng)] * 3
    mask, _ = all_masks(p, 1, old, [70] * 3)
    q = rounded(b.rng.normal(0, 1.5, (90, 4, 64)), BF16)
    tab = b.tab.copy()
    tab[0, 1] = b.pages + 5                  # in the context: every node
    tab[1, 4] = -3                           # tokens 64 .. 79: nodes 24 .. of a star, each seen by itself alone
    args = (dev(q, BF16), dev(tab), dev(np.array([70] * 3, np.int32)), offsets(nodes), as_mask(mask))
    out = host(rg.kv8_tree_attention(b.cache, *args))
    assert np.isnan(out[:30]).all() and np.isnan(out[54:60]).all()
    at = np.r_[30:54, 60:90]
    ref = host(rg.kv8_tree_attention(b.cache, args[0], dev(b.tab), *args[2:]))
    assert np.array_equal(out[at], ref[at])
    # a table that ends inside the tree, and one that has not the sequence's row
    short = dev(np.ascontiguousarray(b.tab[:, :4]))                      # 64 tokens
    out = host(rg.kv8_tree_attention(b.cache, args[0], short, *args[2:]))
    for s in range(3):
        assert np.isnan(out[30 * s + 24:30 * s + 30]).all() and np.array_equal(out[30 * s:30 * s + 24], ref[30 * s:30 * s + 24])
    out = host(rg.kv8_tree_attention(b.cache, args[0], dev(b.tab), *args[2:], tab_row=dev(np.array([0, 9, 2], np.int32))))
    assert np.isnan(out[30:60]).all() and np.array_equal(out[60:], ref[60:])
    # lengths past everything
    n = dev(np.array([70, 2 ** 31 - 1, 70], np.int32))
    out = host(rg.kv8_tree_attention(b.cache, args[0], dev(b.tab), n, *args[3:]))
    assert np.isnan(out[30:60]).all() and np.array_equal(out[60:], ref[60:])


def test_output_in_the_queries_place():
    import paper_2606_02218_amd as rg
    for old in (50, 4000):
        b = Batch([old + 20], 2, 128, 16, seed=old)
        mask, _ = tree.masks(parents(20, "tree", b.rng), 1, old)
        q = dev(rounded(b.rng.normal(0, 1.5, (20, 12, 128)), BF16), BF16)
        args = (dev(b.tab), dev(b.lengths()), offsets([20]), as_mask(mask))
        want = rg.kv8_tree_attention(b.cache, q, *args)
        assert torch.equal(rg.kv8_tree_attention(b.cache, q, *args, out=q), want) and torch.equal(q, want)


# ---------------------------------------------------------------- wide trees over long contexts: 32 columns a workgroup
LONG = 1 << 14                # a bound that asks for them, in chunks, whatever the lengths


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd,n_kv,rep,nodes,old", [
    (128, 1, 7, [64, 64], [9001, 37]), (128, 2, 7, [90, 1, 64], [100, 600, 2050]), (64, 2, 8, [64, 33, 0, 40], [0, 63, 7, 1200]),
    (64, 1, 33, [33, 0, 17, 40], [7, 9, 100, 200]), (128, 1, 128, [5, 1, 9], [0, 63, 64]), (64, 1, 1, [512], [5000]),
    (128, 1, 1, [300], [0]), (64, 3, 6, [65, 128, 3], [129, 0, 3000])])
def test_wide_trees_over_long_contexts(hd, n_kv, rep, nodes, old, dtype):
    import paper_2606_02218_amd as rg
    assert sum(nodes) * rep / len(nodes) > 255
    b = Batch([a + c for a, c in zip(nodes, old)], n_kv, hd, 16 if rep % 2 else 64, seed=hd + rep)
    trees = [parents(n, "tree", b.rng) if n else np.zeros(0, int) for n in nodes]
    mask, _ = all_masks(trees, words_of(nodes), old, b.lengths())
    q = rounded(b.rng.normal(0, 1.5, (sum(nodes), n_kv * rep, hd)), dtype)
    args = (b.cache, dev(q, dtype), dev(b.tab), dev(b.lengths()), offsets(nodes), as_mask(mask))
    for bound in (LONG, 1 << 19):
        out = rg.kv8_tree_attention(*args, max_len=bound)
        check(b, q, nodes, mask, out, dtype)
        assert all(torch.equal(out, rg.kv8_tree_attention(*args, max_len=bound)) for _ in range(2))
    check(b, q, nodes, mask, rg.kv8_tree_attention(*args, max_len=LONG, scale=0.05), dtype, 0.05)


def test_wide_trees_any_mask_padding_and_rows_of_nobody():
    import paper_2606_02218_amd as rg
    nodes, lens = [40, 9, 130, 60], [40, 4, 150, 0]              # 5 rows of the second are padding, all of the last
    b = Batch(lens, 2, 64, 32, seed=5)
    rows = sum(nodes) + 6
    mask = b.rng.integers(0, 2 ** 63, (rows, 3)).astype(np.uint64) * np.uint64(2) + np.uint64(1)
    mask[::5] = 0                                       # with no context these rows see nothing
    mask[1::7] = np.uint64(2 ** 64 - 1)
    q = rounded(b.rng.normal(0, 1.5, (rows, 10, 64)), BF16)
    for words in (3, 1):
        for cut in (0, -7):
            n = b.lengths()
            n[3] = cut
            m = np.ascontiguousarray(mask[:, :words])
            out = torch.full((rows, 10, 64), 9.0, device="cuda", dtype=BF16)
            rg.kv8_tree_attention(b.cache, dev(q, BF16), dev(b.tab), dev(n), offsets(nodes), as_mask(m), out=out, max_len=LONG)
            check(b, q, nodes, m, out, BF16)
            got = host(out)
            assert (got[-6:] == 9.0).all() and not got[179:239].any() and not got[40:45].any()
            assert not got[[i for i in range(40) if i % 5 == 0 and i % 7 != 1]].any()


@pytest.mark.parametrize("old", [45, 3000])
def test_wide_trees_what_a_node_does_not_see(old):
    """NaN codes in nodes, and pages outside the pool and the table."""
    import paper_2606_02218_amd as rg
    n, hd = 40, 64
    b = Batch([old + n], 1, hd, 16, seed=8)
    p = parents(n, "tree", b.rng)
    mask, _ = tree.masks(p, 1, old)
    q = rounded(b.rng.normal(0, 1.5, (n, 8, hd)), BF16)
    args = (dev(q, BF16), dev(b.tab), dev(b.lengths()), offsets([n]), as_mask(mask))
    clean = host(rg.kv8_tree_attention(b.cache, *args, max_len=LONG))
    page, sub = b.places(0, -(-(old + n) // 16))
    v, k = b.cache.v.view(torch.uint8), b.cache.k.view(torch.uint8)
    sees = tree.seen(mask, old + n, n)
    t = old + 11
    for d in (5, 33):
        v[int(page[t // 16]), 0, int(sub[t // 16]), (t % 16 // 4) * 4 * hd + d * 4 + t % 4] = 0x7F
    out = host(rg.kv8_tree_attention(b.cache, *args, max_len=LONG))
    rest = [d for d in range(hd) if d not in (5, 33)]
    for i in range(n):
        if sees[i, t]:
            assert np.isnan(out[i][:, [5, 33]]).all() and np.array_equal(out[i][:, rest], clean[i][:, rest])
        else:
            assert np.array_equal(out[i], clean[i]), i
    t = old + 7
    k[int(page[t // 16]), 0, int(sub[t // 16]), (t % 16) * 16 + 9] = 0xFF
    out2 = host(rg.kv8_tree_attention(b.cache, *args, max_len=LONG))
    for i in range(n):
        assert np.isnan(out2[i]).all() if sees[i, t] else np.array_equal(out2[i], out[i], equal_nan=True), i
    for lost in (b.pages + 5, -3):
        tab = b.tab.copy()
        tab[0, (old + 30) // 16] = lost
        hit = sees[:, (old + 30) // 16 * 16:(old + 30) // 16 * 16 + 16].any(1)
        out3 = host(rg.kv8_tree_attention(b.cache, args[0], dev(tab), *args[2:], max_len=LONG))
        for i in range(n):
            assert np.isnan(out3[i]).all() if hit[i] else np.array_equal(out3[i], out2[i], equal_nan=True), i


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n_kv,rep,old,bound,pieces", [(24, 11, 45, 1000, 1), (24, 11, 3000, 1 << 14, 1), (3, 11, 3000, 3300, 2)])
def test_32_columns_what_a_node_does_not_see(n_kv, rep, old, bound, pieces, hd, dtype):
    """The 32-column kernel, as its plan says: NaN codes that some nodes see, pages outside the pool and the table in
    the tree and in the context, tables that end early or lack the sequence, lengths past everything."""
    import paper_2606_02218_amd as rg
    n, far = 70, 2                                       # the tree in question, and a second sequence beside it
    nodes, olds = [n, n], [old, 31]
    b = Batch([c + n for c in olds], n_kv, hd, 16, capacity=old + n + 60, seed=old + hd)
    wide, cut = cuts(b, n_kv * rep, nodes, far, bound, dtype)
    assert wide and min(cut, 2) == pieces
    trees = [parents(n, "tree", b.rng) for _ in nodes]
    mask, _ = all_masks(trees, far, olds, b.lengths())
    q = rounded(b.rng.normal(0, 1.5, (2 * n, n_kv * rep, hd)), dtype)
    args = (dev(q, dtype), dev(b.tab), dev(b.lengths()), offsets(nodes), as_mask(mask))
    run = lambda tab=args[1], lens=args[2], **k: host(rg.kv8_tree_attention(  # noqa: E731
        b.cache, args[0], tab, lens, *args[3:], max_len=bound, **k))
    clean = run()
    if n_kv * rep < 40:
        check(b, q, nodes, mask, torch.from_numpy(clean), dtype)
    sees = tree.seen(mask[:n], old + n, n)
    page, sub = b.places(0, -(-(old + n) // 16))
    v, k = b.cache.v.view(torch.uint8), b.cache.k.view(torch.uint8)
    h, here = 1, slice(rep, 2 * rep)                     # the kv head with bad codes, its query heads
    t = old + 11
    for d in (5, hd - 31):
        v[int(page[t // 16]), h, int(sub[t // 16]), (t % 16 // 4) * 4 * hd + d * 4 + t % 4] = 0x7F
    want = clean.copy()
    for d in (5, hd - 31):
        want[:n, here, d] = np.where(sees[:, t, None], np.nan, want[:n, here, d])
    assert sees[:, t].any() and not sees[:, t].all()
    assert np.array_equal(run(), want, equal_nan=True)
    t = old + 67
    k[int(page[t // 16]), h, int(sub[t // 16]), (9 // 16) * 256 + (t % 16) * 16 + 9] = 0xFF
    want[:n, here] = np.where(sees[:, t, None, None], np.nan, want[:n, here])
    assert np.array_equal(run(), want, equal_nan=True)
    for lost, t in ((b.pages + 5, old + 20), (-3, old + 66), (2 ** 31 - 1, old - 40), (b.pages, 3)):
        tab = b.tab.copy()
        tab[0, t // 16] = lost
        hit = sees[:, t // 16 * 16:t // 16 * 16 + 16].any(1)
        bad = want.copy()
        bad[:n][hit] = np.nan
        assert np.array_equal(run(dev(tab)), bad, equal_nan=True), t
    short = (old + 40) // 16                             # pages of a table that ends inside the tree
    bad = want.copy()
    bad[:n][sees[:, short * 16:].any(1)] = np.nan
    bad[n:][tree.seen(mask[n:], 31 + n, n)[:, short * 16:].any(1)] = np.nan
    assert np.array_equal(run(dev(np.ascontiguousarray(b.tab[:, :short]))), bad, equal_nan=True)
    bad = want.copy()
    bad[:n] = np.nan
    assert np.array_equal(run(tab_row=dev(np.array([9, 1], np.int32))), bad, equal_nan=True)
    assert np.array_equal(run(lens=dev(np.array([2 ** 31 - 1, 31 + n], np.int32))), bad, equal_nan=True)


def test_wide_trees_in_the_queries_place():
    import paper_2606_02218_amd as rg
    for old, bound in ((50, LONG), (4000, LONG), (50, 8192)):
        b = Batch([old + 30], 2, 128, 16, seed=old)
        mask, _ = tree.masks(parents(30, "tree", b.rng), 1, old)
        q = dev(rounded(b.rng.normal(0, 1.5, (30, 28, 128)), BF16), BF16)
        args = (dev(b.tab), dev(b.lengths()), offsets([30]), as_mask(mask))
        want = rg.kv8_tree_attention(b.cache, q, *args, max_len=bound)
        assert torch.equal(rg.kv8_tree_attention(b.cache, q, *args, out=q, max_len=bound), want) and torch.equal(q, want)


# ---------------------------------------------------------------- accepted paths
def accepted(b, nodes, old, trees, last, words):
    """The oracle's caches after the accept; its lengths."""
    out = []
    for s, (n, c, p, i) in enumerate(zip(nodes, old, trees, last)):
        keep = tree.paths(p, max(-c, 0))[i] if 0 <= i < n else []
        keep = [j for j in keep or [] if j < 64 * words]
        m = [tree.accept(x[s], max(c, 0), keep, max(-c, 0)) for x in (b.k, b.v)]
        out.append(m[0])
    return np.array(out, np.int32)


@pytest.mark.parametrize("kind", ["chain", "star", "forest", "tree"])
@pytest.mark.parametrize("hd,n_kv,page", [(64, 3, 16), (128, 2, 64)])
def test_accept(kind, hd, n_kv, page):
    """Codes and scales bit for bit, of every block: those that received tokens and all the others."""
    import paper_2606_02218_amd as rg
    nodes = [1, 5, 40, 64, 0, 17, 33, 8, 90, 250]
    old = [0, 3, 15, 16, 50, 31, 7, 200, 1, 29]
    words = 4
    b = Batch([0] * len(nodes), n_kv, hd, page, capacity=400, seed=hd + len(kind))
    for s, (n, c) in enumerate(zip(nodes, old)):
        for x in (b.k, b.v):                 # magnitudes over many octaves: scales differ from block to block
            a = b.rng.normal(0, 1, (n + c, n_kv, hd)) * np.exp2(b.rng.integers(-12, 9, (n + c, n_kv, 1)))
            if n + c:
                x[s].append(rounded(a, F32))
    b.write()
    trees = [parents(n, kind, b.rng) if n else np.zeros(0, int) for n in nodes]
    last = [int(b.rng.integers(0, n)) if n else -1 for n in nodes]
    last[2], last[7] = 39, -1
    mask, _ = all_masks(trees, words, old, b.lengths())
    lens = b.lengths()
    before = b.snapshot()
    new = rg.kv8_accept(b.cache, dev(b.tab), dev(lens), offsets(nodes), as_mask(mask), dev(np.array(last, np.int32)))
    want = accepted(b, nodes, old, trees, last, words)
    assert np.array_equal(new.cpu().numpy(), want)
    # slots behind the end keep what they hold: the oracle's caches hold them too
    image = [x.copy() for x in before]
    for s in range(len(nodes)):
        for (codes, scales), seq, keys in (((0, 1), b.k[s], True), ((2, 3), b.v[s], False)):
            c, m = b.blocks(seq, keys)
            pg, sub = b.places(s, len(c))
            image[codes][pg, :, sub] = np.where(m, c, image[codes][pg, :, sub])
            image[scales][pg, :, sub] = seq.scale[:len(c)]
    for got, ref in zip(b.snapshot(), image):
        assert np.array_equal(got, ref)


def test_accept_of_padding_lost_pages_and_numbers_out_of_range():
    import paper_2606_02218_amd as rg
    hd = 64
    b = Batch([40, 40, 6, 40, 40], 1, hd, 16, capacity=48, seed=2)
    nodes, old = [20, 20, 10, 20, 20], [20, 20, -4, 20, 20]
    trees = [np.array([-1] + [max(0, i - 2) for i in range(1, n)]) for n in nodes]
    mask, _ = all_masks(trees, 1, [max(c, 0) for c in old], b.lengths())
    tab, last = b.tab.copy(), [19, 40, 9, 19, -5]
    tab[3, 2] = -1                           # tokens 32 ..: sources are lost
    before = b.snapshot()
    new = rg.kv8_accept(b.cache, dev(tab), dev(b.lengths()), offsets(nodes), as_mask(mask), dev(np.array(last, np.int32)))
    kept = tree.paths(trees[3], 0)[19]
    assert new.cpu().tolist() == [20 + len(tree.paths(trees[0])[19]), 20, len(tree.paths(trees[2], 4)[9]), 20 + len(kept), 20]
    after = b.snapshot()
    for s in (1, 4):                         # nothing accepted: nothing touched
        for x, y in zip(before, after):
            assert np.array_equal(x[b.tab[s]], y[b.tab[s]])
    # the accepted tokens from lost pages arrive as NaN, the others as they were
    values = b.logical(3, 20 + len(kept), True)
    was = b.k[3].values()
    for j, i in enumerate(kept):
        if 20 + i >= 32:
            assert np.isnan(values[20 + j]).all()
        else:
            assert np.all(np.abs(values[20 + j] - was[20 + i]) <= 2.0 ** -9 * np.abs(was).max())
    assert np.array_equal(values[:16], was[:16])


def test_accept_keeps_nan():
    import paper_2606_02218_amd as rg
    b = Batch([30], 1, 64, 16, seed=6)
    raw = b.cache.k.view(torch.uint8)
    t = 25
    raw[int(b.tab[0, 1]), 0, 0, (t % 16) * 16 + 3] = 0x7F
    mask, _ = tree.masks([-1, 0, 0, 0, 0, 0, 0, 0, 0, 0], 1, 20)
    rg.kv8_accept(b.cache, dev(b.tab), dev(b.lengths()), offsets([10]), as_mask(mask), dev(np.array([5], np.int32)))
    got = b.logical(0, 22, True)
    assert np.isnan(got[21, 0, 3]) and np.isnan(got[:21]).sum() == 0 and np.isnan(got[21]).sum() == 1


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("graph", [False, True])
def test_a_round_of_drafting(graph):
    """Positions, turned keys, append, attention, draw, the accepted path and its move, as a program runs them; then
    the next token over the moved cache.  Eagerly and replayed from a graph."""
    import paper_2606_02218_amd as rg
    n_kv, rep, hd, vocab, nodes = 2, 3, 64, 500, [7, 12, 1, 20]
    old = [30, 5, 100, 64]
    rows = sum(nodes)
    b = Batch(old, n_kv, hd, 16, capacity=160, seed=11)
    rng = b.rng
    trees = [parents(n, "tree", rng) for n in nodes]
    draft = rng.integers(0, vocab, rows).astype(np.int32)
    off, tab = offsets(nodes), dev(b.tab)
    seq_len = dev((np.array(old) + nodes).astype(np.int32))
    cos, sin = rg.rope_table(400, hd)
    q, k, v = (rounded(rng.normal(0, 1, (rows, h, hd)), BF16) for h in (n_kv * rep, n_kv, n_kv))
    dq, dk, dv = dev(q, BF16), dev(k, BF16), dev(v, BF16)
    head = rng.normal(0, 0.3, (n_kv * rep * hd, vocab))
    u = dev(rng.random(rows).astype(np.float32))
    parent = dev(np.concatenate(trees).astype(np.int32))
    dh, ddraft = dev(head, F32), dev(draft)
    seq = dev(np.repeat(np.arange(len(nodes)), nodes))

    def step():
        mask, pos = rg.kv8_tree(parent, seq_len, off)
        tq, tk = rg.rope(dq, pos, cos, sin), rg.rope(dk, pos, cos, sin)
        rg.kv8_append(b.cache, tk, dv, tab, seq_len, off)
        att = rg.kv8_tree_attention(b.cache, tq, tab, seq_len, off, mask)
        logits = att.float().view(rows, -1) @ dh
        token, lp, kept = rg.sample(logits, u, temperature=0.8, top_k=40, top_p=0.9)
        # a node is accepted if its parent drew it; the last accepted one is the deepest
        up = (off[:-1].long()[seq] + parent.long()).clamp(min=0)
        right = (parent < 0) | (token[up] == ddraft)
        bits = right.long() << (torch.arange(rows, device="cuda") - off[:-1].long()[seq])
        ok = torch.zeros(len(nodes), dtype=torch.int64, device="cuda").index_add_(0, seq, bits)[seq]
        depth = torch.where((mask[:, 0] & ~ok) == 0, pos, -1)
        best = torch.full((len(nodes),), -1, dtype=torch.int32, device="cuda").scatter_reduce(0, seq, depth, "amax")
        number = (torch.arange(rows, device="cuda") - off[:-1].long()[seq]).int()
        last = torch.full((len(nodes),), 1 << 20, dtype=torch.int32, device="cuda").scatter_reduce(
            0, seq, torch.where(depth == best[seq], number, 1 << 20).int(), "amin")
        new_len = rg.kv8_accept(b.cache, tab, seq_len, off, mask, last)
        return mask, pos, att, logits, token, lp, kept, last, new_len

    start = [t.clone() for t in b.cache]

    def reset():
        for t, x in zip(b.cache, start):
            t.view(torch.uint8).copy_(x.view(torch.uint8))

    got = [x.clone() for x in step()]
    after = [t.clone() for t in b.cache]
    if graph:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = step()
        for _ in range(3):
            reset()
            for x in outs:
                x.zero_()
            g.replay()
            torch.cuda.synchronize()
            for x, y in zip(outs, got):
                assert torch.equal(x, y)
            for t, x in zip(b.cache, after):
                assert torch.equal(t.view(torch.uint8), x.view(torch.uint8))
    mask, pos, att, logits, token, lp, kept, last, new_len = (x.cpu().numpy() if x.dtype != BF16 else host(x) for x in got)
    # the oracle's round
    want, at = all_masks(trees, 1, old, np.array(old) + nodes)
    assert np.array_equal(mask.view(np.uint64), want) and np.array_equal(pos, at)
    c, s = cos.cpu().numpy()[at], sin.cpu().numpy()[at]
    tq = host(rg.rope(dq, dev(at.astype(np.int32)), cos, sin))
    tk = host(rg.rope(dk, dev(at.astype(np.int32)), cos, sin))
    assert np.allclose(tk, kv8.rotate(k, c, s), rtol=2.0 ** -8, atol=1e-6)
    for i, n in enumerate(nodes):
        r = slice(sum(nodes[:i]), sum(nodes[:i + 1]))
        b.k[i].append(tk[r])
        b.v[i].append(v[r])
    check(b, tq, nodes, want, torch.from_numpy(att), BF16)
    for i, n in enumerate(nodes):
        r0 = sum(nodes[:i])
        good = [j == 0 or token[r0 + trees[i][j]] == draft[r0 + j] for j in range(n)]
        paths = tree.paths(trees[i])
        ends = [j for j in range(n) if all(good[a] for a in paths[j])]
        deepest = max(len(paths[j]) for j in ends)
        assert last[i] == min(j for j in ends if len(paths[j]) == deepest)
        m = tree.accept(b.k[i], old[i], paths[last[i]])
        assert tree.accept(b.v[i], old[i], paths[last[i]]) == m == new_len[i]
    # the next token's attention over what is left
    x = rounded(rng.normal(0, 1.5, (len(nodes), n_kv * rep, hd)), BF16)
    for t, y in zip(b.cache, after):
        t.view(torch.uint8).copy_(y.view(torch.uint8))
    out = host(rg.kv8_attention(b.cache, dev(x, BF16), tab, dev(new_len.astype(np.int32))))
    for i in range(len(nodes)):
        n = int(new_len[i])
        ref, mass, reach = kv8.attend(x[i:i + 1], b.k[i].values()[:n], b.v[i].values()[:n], [n - 1], hd ** -0.5)
        bound = attention_bound(ref, mass, reach, hd, n, hd ** -0.5, BF16, 2.0 ** -16)
        assert np.all(np.abs(out[i:i + 1] - ref) <= bound)


def test_streams():
    """A call on a given stream, and two calls at once on two streams: same bits."""
    import paper_2606_02218_amd as rg
    b = Batch([3000, 70], 2, 128, 16, seed=12)
    nodes = [40, 30]
    trees = [parents(n, "tree", b.rng) for n in nodes]
    parent, off, n = dev(np.concatenate(trees).astype(np.int32)), offsets(nodes), dev(b.lengths())
    q = dev(rounded(b.rng.normal(0, 1.5, (70, 12, 128)), BF16), BF16)
    mask, pos = rg.kv8_tree(parent, n, off)
    want = rg.kv8_tree_attention(b.cache, q, dev(b.tab), n, off, mask)
    tab = dev(b.tab)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        outs = []
        for s in streams:
            m, p = rg.kv8_tree(parent, n, off, stream=s)
            outs.append((m, p, rg.kv8_tree_attention(b.cache, q, tab, n, off, m, stream=s)))
        torch.cuda.synchronize()
        for m, p, x in outs:
            assert torch.equal(m, mask) and torch.equal(p, pos) and torch.equal(x, want)
