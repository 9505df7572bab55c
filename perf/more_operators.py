"""Decoding with drafted trees over the 8-bit paged cache, and a truncated
sampler: their calls as cases to be timed and checked.

Four operators: ``kv8_tree`` (what each drafted token sees of its tree, and its
position), ``kv8_tree_attention`` (attention of the drafted tokens over the cache
and their own ancestors), ``kv8_accept`` (the accepted path takes its place in the
cache) and ``sample`` (temperature, top-k, top-p and min-p from given random
numbers).  ``run`` computes each in elementary torch operations, or, with ``own``
set, by the library's entry points.

The cache.  16 consecutive tokens of one kv head are a block with one scale, a
power of two; a page is page_tokens / 16 blocks of every kv head, a sequence a
row of page ids.  A value is an e4m3 code times its block's scale.  Inside a
block, keys lie as [dim / 16][token][dim % 16], values as
[token / 4][dim][token % 4].

A tree.  A sequence's last n tokens are drafted nodes, each behind its parent; a
node's mask holds a bit for itself and each ancestor.  Node i lies in slot
context + i of the cache and at position context + depth.

Accept.  The nodes of a mask move to the slots behind the context, in their order.
A block that receives one takes the largest scale among the tokens that end up in
it; their codes are rounded again to nearest even where theirs was smaller.

Sampling.  Weights are exp((z - max z) / T).  Tokens in order of z, ties by id:
top-k keeps the first k, top-p those before which less than p of the k's weight
lies, min-p those of at least min_p of the largest weight.  The token drawn is the
first, by id, at which the kept weights' running sum passes u of their sum.
"""
import math
import random

import torch

own = False

# (query heads, kv heads, head_dim) of the repository's bf16 workloads, and their vocabularies
_HEADS = {"gpt2s": (12, 12, 64), "1.5b": (12, 2, 128), "7b": (28, 4, 128)}
_VOCAB = {"gpt2s": 32000, "1.5b": 151936, "7b": 152064}
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _tree(seqs, nodes, shape="tree", name=None):
    c = {"name": name} if name else {}
    c.update(kind="tree", seqs=seqs, nodes_lo=nodes[0], nodes_hi=nodes[1], old_lo=100, old_hi=4000, shape=shape)
    return c


def _attend(model, seqs, nodes, old, dtype, shape="tree", page=16, name=None):
    """nodes, old: (lo, hi) drafted tokens of a sequence and tokens that it holds before them."""
    c = {"name": name} if name else {}
    c.update(kind="attend", model=model, seqs=seqs, nodes_lo=nodes[0], nodes_hi=nodes[1], old_lo=old[0], old_hi=old[1],
             dtype=dtype, shape=shape, page=page)
    return c


def _accept(model, seqs, nodes, old, shape="tree", page=16, name=None):
    c = {"name": name} if name else {}
    c.update(kind="accept", model=model, seqs=seqs, nodes_lo=nodes[0], nodes_hi=nodes[1], old_lo=old[0], old_hi=old[1],
             shape=shape, page=page)
    return c


def _sample(rows, vocab, dtype, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, by_row=False, name=None):
    """by_row: a temperature, k, p and min-p for every row, spread around the ones given."""
    c = {"name": name} if name else {}
    c.update(kind="sample", rows=rows, vocab=vocab, dtype=dtype, temperature=temperature, top_k=top_k, top_p=top_p,
             min_p=min_p, by_row=by_row)
    return c


def listed():
    return [
        # A handful of sequences with small trees: latency only.
        _tree(8, (5, 16), name="tree_step_8"),
        # A large serving batch with wide, ragged trees.
        _tree(509, (17, 64), name="tree_batch_509"),
        # Few sequences of the small model: latency.
        _attend("gpt2s", 8, (8, 16), (200, 600), "bf16", name="attend_tree_gpt2s"),
        # A serving batch at ordinary contexts, ragged trees.
        _attend("1.5b", 64, (4, 63), (512, 4500), "bf16", name="attend_tree_1.5b"),
        # Two very long contexts: the work of each has to be split.
        _attend("7b", 2, (64, 64), (60001, 131000), "bf16", page=64, name="attend_tree_long_7b"),
        # fp32 queries, trees of more nodes than one 64-bit mask holds.
        _attend("1.5b", 23, (65, 200), (131, 2000), "f32", page=32, name="attend_wide_trees_f32"),
        # A handful of sequences: latency.
        _accept("gpt2s", 8, (8, 16), (200, 600), name="accept_gpt2s"),
        # A large batch; long accepted chains that cross blocks.
        _accept("7b", 256, (33, 64), (100, 1200), shape="deep", page=64, name="accept_deep_7b"),
        # The last sequences of a batch, a narrow sampler.
        _sample(8, 151936, "bf16", 0.7, 20, 0.8, name="sample_tail_1.5b"),
        # A full training batch: every token can be drawn.
        _sample(512, 151936, "f32", 1.0, name="sample_step_1.5b"),
        # A nucleus alone, from one token to many thousands by the row.
        _sample(64, 152064, "bf16", 1.0, 0, 0.95, name="sample_nucleus_7b"),
        # A serving batch where each request has its own settings.
        _sample(505, 32000, "bf16", 0.9, 50, 0.9, 0.05, by_row=True, name="sample_by_row_gpt2s"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: sizes log-uniform, odd ones among them."""
    kind = rng.choice(["tree", "attend", "attend", "attend long", "accept", "sample", "sample", "sample"])
    model = rng.choice(sorted(_HEADS))
    shape, page = rng.choice(["tree", "tree", "deep", "wide"]), rng.choice([16, 16, 32, 64])
    lo = _log_int(rng, 1, 40)
    nodes = (lo, lo + _log_int(rng, 1, 25) - 1)
    if kind == "tree":
        return _tree(_log_int(rng, 1, 512), nodes, shape)
    if kind == "attend":
        n, seqs = _log_int(rng, 1, 1500), _log_int(rng, 1, 48)
        if rng.random() < 0.2:
            nodes, seqs = (66, 66 + _log_int(rng, 1, 120)), min(seqs, 15)
        return _attend(model, seqs, nodes, (n, n + rng.randint(0, 800)), rng.choice(["bf16", "bf16", "f32"]), shape, page)
    if kind == "attend long":
        n = _log_int(rng, 4000, 40000)
        return _attend(rng.choice(["1.5b", "7b"]), rng.randint(1, 3), nodes, (n, n + rng.randint(0, n // 4)), "bf16", shape,
                       page)
    if kind == "accept":
        n = _log_int(rng, 1, 1000)
        return _accept(model, _log_int(rng, 1, 256), nodes, (n, n + rng.randint(0, 400)), shape, page)
    vocab = _VOCAB[model] if rng.random() < 0.5 else _log_int(rng, 200, 160000)
    return _sample(_log_int(rng, 1, 512), vocab, rng.choice(["bf16", "f32"]), round(rng.uniform(0.5, 1.3), 2),
                   rng.choice([0, 0, _log_int(rng, 1, 300)]), rng.choice([1.0, round(rng.uniform(0.5, 0.99), 3)]),
                   rng.choice([0.0, 0.0, round(rng.uniform(0.01, 0.2), 3)]), rng.random() < 0.3)


# ---------------------------------------------------------------- inputs
def _rng_of(case):
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _lengths(case):
    """(drafted nodes, tokens held before them) of every sequence; they follow from the case alone."""
    r = _rng_of(case)
    new = [r.randint(case["nodes_lo"], case["nodes_hi"]) for _ in range(case["seqs"])]
    return new, [r.randint(case["old_lo"], case["old_hi"]) for _ in range(case["seqs"])]


def _words(case):
    return (case["nodes_hi"] + 63) // 64


def _parents(case, seed):
    """Each node's parent among its sequence's nodes.  Node 0 is the last token that was emitted, whose successors were
    drafted: deep trees are chains with a few branches, wide ones mostly leaves."""
    r = random.Random(seed * 31 + 5)
    back = {"tree": 4, "deep": 1, "wide": 64}[case["shape"]]
    out = []
    for n in _lengths(case)[0]:
        out += [-1] + [max(0, i - 1 - r.randint(0, back) * (r.random() < 0.5)) for i in range(1, n)]
    return torch.tensor(out, device="cuda", dtype=torch.int32)


def _last(case, seed):
    """The last accepted node of every sequence: mostly some node, now and then none."""
    r = random.Random(seed * 17 + 3)
    return torch.tensor([r.randint(-1, n - 1) for n in _lengths(case)[0]], device="cuda", dtype=torch.int32)


def _pages(case, gen):
    """A page table of scattered pages and the number of pages of the pool."""
    new, old = _lengths(case)
    pt = case["page"]
    need = torch.tensor([(a + b + pt - 1) // pt for a, b in zip(new, old)], device="cuda")
    width, total = int(need.max()), int(need.sum())
    pool = total + 3                                                # a pool holds pages of nobody too
    tab = torch.zeros(case["seqs"], width, dtype=torch.int64, device="cuda")
    tab[torch.arange(width, device="cuda") < need[:, None]] = torch.randperm(pool, generator=gen, device="cuda")[:total]
    return tab.int(), pool


def _pool(case, pool, gen):
    """A cache as earlier appends left it: codes of all sizes and scales of a few octaves."""
    _, nkv, hd = _HEADS[case["model"]]
    m = case["page"] // 16

    def codes():
        c = torch.empty(pool, nkv, m, 16 * hd, device="cuda", dtype=torch.float8_e4m3fn)
        step = max(1, (1 << 26) // (nkv * m * 16 * hd))
        for a in range(0, pool, step):
            part = c[a:a + step]
            c[a:a + step] = (torch.randn(part.shape, generator=gen, device="cuda") * 90.0).clamp(-448.0, 448.0).to(c.dtype)
        return c

    def scales():
        return torch.exp2(torch.randint(-8, -5, (pool, nkv, m), generator=gen, device="cuda").float())

    return codes(), codes(), scales(), scales()


def _logits(case, gen):
    """Logits as a decoder gives them: most tokens around nothing, some dozens far above, by how much depends on the row."""
    rows, v = case["rows"], case["vocab"]
    z = 2.0 * torch.randn(rows, v, generator=gen, device="cuda")
    n = min(40, v)
    at = torch.randint(0, v, (rows, n), generator=gen, device="cuda")
    top = 10.0 + 10.0 * torch.rand(rows, 1, generator=gen, device="cuda")
    z.scatter_reduce_(1, at, top - 9.0 * torch.rand(rows, n, generator=gen, device="cuda"), "amax")
    return z.to(_DT[case["dtype"]])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 11)
    if case["kind"] == "sample":
        n = case["rows"]
        st = {"case": case, "z": _logits(case, gen), "u": torch.rand(n, generator=gen, device="cuda")}
        one = {"temperature": case["temperature"], "top_k": case["top_k"], "top_p": case["top_p"], "min_p": case["min_p"]}
        if case["by_row"]:
            f = torch.rand(4, n, generator=gen, device="cuda")
            one = {"temperature": one["temperature"] * (0.5 + f[0]),
                   "top_k": torch.where(f[1] < 0.2, 0, (f[1] * 2 * one["top_k"]).int() + 1).int(),
                   "top_p": (one["top_p"] + 0.4 * (f[2] - 0.5)).clamp(0.1, 1.0), "min_p": one["min_p"] * 2 * f[3]}
        return {**st, "opts": one}
    new, old = _lengths(case)
    st = {"case": case, "off": torch.tensor([0] + new, device="cuda").cumsum(0).int(), "parent": _parents(case, seed),
          "len": torch.tensor([a + b for a, b in zip(new, old)], device="cuda", dtype=torch.int32)}
    if case["kind"] == "tree":
        return st
    st["mask"] = _plain_tree(st)["mask"]
    st["tab"], pool = _pages(case, gen)
    st["cache"], st["max_len"] = _pool(case, pool, gen), max(a + b for a, b in zip(new, old))
    if case["kind"] == "accept":
        st["last"] = _last(case, seed)
    else:
        nq, _, hd = _HEADS[case["model"]]
        st["q"] = (1.5 * torch.randn(sum(new), nq, hd, generator=gen, device="cuda")).to(_DT[case["dtype"]])
    return st


# ---------------------------------------------------------------- the plain form
def _places(state):
    """Of every row: its sequence, its number among the sequence's nodes, the tokens before the tree."""
    off = state["off"].long()
    n = off[1:] - off[:-1]
    seq = torch.repeat_interleave(torch.arange(n.numel(), device="cuda"), n, output_size=state["parent"].numel())
    return seq, torch.arange(seq.numel(), device="cuda") - off[seq], (state["len"].long() - n)


def _plain_tree(state):
    """Ancestors as the closure of "is the parent of", by squaring."""
    case = state["case"]
    n, words = case["nodes_hi"], _words(case)
    seq, node, ctx = _places(state)
    up = torch.zeros(case["seqs"], n, n, device="cuda")
    up[:, torch.arange(n, device="cuda"), torch.arange(n, device="cuda")] = 1.0
    child = state["parent"] >= 0
    up[seq[child], node[child], state["parent"].long()[child]] = 1.0
    for _ in range(max(1, n - 1).bit_length()):
        up = torch.bmm(up, up).clamp_(max=1.0)
    sees = torch.nn.functional.pad(up[seq, node], (0, 64 * words - n)).long()
    mask = (sees.view(-1, words, 64) << torch.arange(64, device="cuda")).sum(-1)
    return {"mask": mask, "pos": (ctx[seq] + sees.sum(-1) - 1).int()}


def _bits(mask):
    """[rows, 64 words] truth values of a mask's bits."""
    return ((mask[:, :, None] >> torch.arange(64, device="cuda")) & 1).flatten(1).bool()


def _gathered(codes, scale, tab, hd, keys):
    """fp32 [sequences, kv heads, tokens, hd] of the pages of a table."""
    c = codes.view(torch.uint8)[tab].view(codes.dtype)               # [S, pages, nkv, m, 16 * hd]
    S, n, nkv, m, _ = c.shape
    if keys:
        c = c.view(S, n, nkv, m, hd // 16, 16, 16).permute(0, 2, 1, 3, 5, 4, 6)
    else:
        c = c.view(S, n, nkv, m, 4, hd, 4).permute(0, 2, 1, 3, 4, 6, 5)
    c = c.reshape(S, nkv, n, m, 16, hd).float()
    return c.mul_(scale[tab].permute(0, 2, 1, 3)[..., None, None]).reshape(S, nkv, n * m * 16, hd)


def _plain_attend(state):
    case = state["case"]
    nq, nkv, hd = _HEADS[case["model"]]
    rep = nq // nkv
    kc, vc, ks, vs = state["cache"]
    seq, node, ctx = _places(state)
    S, L, R = case["seqs"], state["max_len"], case["nodes_hi"]
    tab = state["tab"].long()
    at = torch.arange(L, device="cuda")
    seen = torch.zeros(S, R, L, dtype=torch.bool, device="cuda")
    j = at - ctx[seq][:, None]                                       # [rows, L]: the node that a token is
    bits = _bits(state["mask"])
    seen[seq, node] = (j < 0) | (bits.gather(1, j.clamp(0, bits.shape[1] - 1)) & (j < bits.shape[1]))
    k = _gathered(kc, ks, tab, hd, True)[:, :, :L]
    q = torch.zeros(S, R, nkv, rep, hd, device="cuda")
    q[seq, node] = state["q"].float().view(-1, nkv, rep, hd)
    s = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(S, nkv, R * rep, hd), k.transpose(2, 3)).mul_(hd ** -0.5)
    del k
    s = s.view(S, nkv, R, rep, L).masked_fill_(~seen[:, None, :, None], -math.inf)
    s.sub_(s.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(S, nkv, R * rep, L), _gathered(vc, vs, tab, hd, False)[:, :, :L]).view(S, nkv, R, rep, hd)
    o = (o / total.clamp(min=1e-30)).permute(0, 2, 1, 3, 4).reshape(S, R, nq, hd)
    return {"out": o[seq, node].to(state["q"].dtype)}


def _plain_accept(state):
    case = state["case"]
    _, nkv, hd = _HEADS[case["model"]]
    m, pt = case["page"] // 16, case["page"]
    off, last, tab = state["off"].long(), state["last"].long(), state["tab"].long()
    ctx = state["len"].long() - (off[1:] - off[:-1])
    keep = _bits(state["mask"][(off[:-1] + last).clamp(min=0)]) & (last >= 0)[:, None]     # [S, nodes]
    new_len = ctx + keep.sum(1)
    seq, node = keep.nonzero(as_tuple=True)
    src = ctx[seq] + node
    dst = ctx[seq] + keep.cumsum(1)[seq, node] - 1
    moved = src != dst
    # every block that receives a token, and the tokens that end up in it: (block, slot, source block, source slot)
    hit = torch.zeros(case["seqs"], tab.shape[1] * m, dtype=torch.bool, device="cuda")
    hit[seq[moved], dst[moved] // 16] = True
    bs, bb = hit.nonzero(as_tuple=True)
    t = bb[:, None] * 16 + torch.arange(16, device="cuda")           # [blocks, 16] positions
    there = t < new_len[bs][:, None]
    where = torch.arange(tab.shape[1] * pt, device="cuda").repeat(case["seqs"], 1)
    where[seq, dst] = src
    fro = torch.where(there, where[bs].gather(1, t), t)
    page = lambda x: tab[bs[:, None], x // pt]  # noqa: E731
    sub = lambda x: x % pt // 16  # noqa: E731
    head = torch.arange(nkv, device="cuda")[None, :, None]
    dim = torch.arange(hd, device="cuda")
    pf, sf, pd, sd = page(fro), sub(fro), page(t), sub(t)
    for codes, scale, keys in ((state["cache"][0], state["cache"][2], True), (state["cache"][1], state["cache"][3], False)):
        pool = codes.shape[0]
        raw = codes.view(torch.uint8)
        view = raw.view(pool, nkv, m, hd // 16, 16, 16) if keys else raw.view(pool, nkv, m, 4, hd, 4)

        def index(p, s, x):
            p, s, x, h = p[:, None, :, None], s[:, None, :, None], x[:, None, :, None] % 16, head[..., None]
            return (p, h, s, dim // 16, x, dim % 16) if keys else (p, h, s, x // 4, dim, x % 4)
        got = view[index(pf, sf, fro)]                               # [blocks, nkv, 16, hd]
        was = scale[pf[:, None], head, sf[:, None]]                  # [blocks, nkv, 16]
        top = torch.where(there[:, None], was, 0.0).amax(-1)
        again = (got.view(codes.dtype).double() * (was / top[..., None])[..., None].double()).float().to(codes.dtype)
        view[index(pd, sd, t)] = torch.where(there[:, None, :, None], again.view(torch.uint8), got)
        scale[pd[:, :1], head[..., 0], sd[:, :1]] = top
    kc, vc, ks, vs = state["cache"]
    return {"k": kc, "v": vc, "k_scale": ks, "v_scale": vs, "len": new_len.int()}


def _column(x, rows):
    """A setting as a column of 64-bit numbers."""
    return x.double()[:, None] if isinstance(x, torch.Tensor) else torch.full((rows, 1), x, dtype=torch.float64, device="cuda")


def _plain_sample(state):
    case, z = state["case"], state["z"]
    rows, v = z.shape
    t, k, p, least = (_column(state["opts"][n], rows) for n in ("temperature", "top_k", "top_p", "min_p"))
    x = z.double()
    top = x.amax(1, keepdim=True)
    w = ((x - top) / t).exp_()
    total = w.sum(1, keepdim=True)
    if case["by_row"] or case["top_k"] or case["top_p"] < 1 or case["min_p"] > 0:
        zs, order = torch.sort(z.float(), dim=1, descending=True, stable=True)
        ws = w.gather(1, order)
        keep = (torch.arange(v, device="cuda") < k) | (k <= 0)
        ws.masked_fill_(~keep, 0.0)
        run = ws.cumsum(1)
        keep &= (run - ws < p * run[:, -1:]) | (p >= 1)
        keep &= zs.double() >= top + t * least.log()
        w = w.masked_fill(~torch.zeros_like(keep).scatter_(1, order, keep), 0.0)
    run = w.cumsum(1)
    tok = (run <= state["u"].double()[:, None] * run[:, -1:]).sum(1, keepdim=True)
    lw = (x.gather(1, tok) - top) / t
    return {"token": tok[:, 0].int(), "logprob": (lw - total.log()).float()[:, 0], "kept": (lw - run[:, -1:].log()).float()[:, 0]}


def run(state):
    case = state["case"]
    if own:
        import paper_2606_02218_amd as rg
        if case["kind"] == "sample":
            token, logprob, kept = rg.sample(state["z"], state["u"], **state["opts"])
            return {"token": token, "logprob": logprob, "kept": kept}
        if case["kind"] == "tree":
            mask, pos = rg.kv8_tree(state["parent"], state["len"], state["off"], words=_words(case))
            return {"mask": mask, "pos": pos}
        cache = rg.Kv8Cache(*state["cache"])
        if case["kind"] == "accept":
            n = rg.kv8_accept(cache, state["tab"], state["len"], state["off"], state["mask"], state["last"])
            return {"k": cache.k, "v": cache.v, "k_scale": cache.k_scale, "v_scale": cache.v_scale, "len": n}
        return {"out": rg.kv8_tree_attention(cache, state["q"], state["tab"], state["len"], state["off"], state["mask"],
                                             max_len=state["max_len"])}
    return {"sample": _plain_sample, "tree": _plain_tree, "accept": _plain_accept, "attend": _plain_attend}[case["kind"]](state)


def _depth(case):
    """About how many nodes a path has."""
    n = (case["nodes_lo"] + case["nodes_hi"]) / 2
    return {"tree": 0.5 * n ** 0.9, "deep": 0.45 * n, "wide": 2.0 + n / 64}[case["shape"]]


def work(case):
    if case["kind"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * (2 if case["dtype"] == "bf16" else 4) + 16 * case["rows"], "flops": 4 * n}
    new, old = _lengths(case)
    rows = sum(new)
    if case["kind"] == "tree":
        return {"bytes": rows * (8 + 8 * _words(case)) + 8 * len(new), "flops": rows * _words(case)}
    nq, nkv, hd = _HEADS[case["model"]]
    if case["kind"] == "accept":
        kept = min(0.5 * _depth(case) * case["seqs"], rows)
        return {"bytes": kept * nkv * 2 * (2 * hd + 1) + 16 * len(new), "flops": kept * nkv * 2 * hd}
    eb = 2 if case["dtype"] == "bf16" else 4
    pairs = sum(a * b for a, b in zip(new, old)) + rows * _depth(case)
    return {"bytes": (rows + sum(old)) * nkv * (2 * hd + 0.5) + rows * (2 * nq * hd * eb + 8 * _words(case)),
            "flops": 4 * hd * nq * pairs}


# ---------------------------------------------------------------- 64 bits
def exact(case, seed):
    with torch.no_grad():
        st = prepare(case, seed)
        return {"sample": _exact_sample, "tree": _exact_tree, "accept": _exact_accept, "attend": _exact_attend}[case["kind"]](case, st, seed)


def _paths(case, seed):
    """Per sequence, each node's ancestors and itself, from the parents alone."""
    parent, out, r = _parents(case, seed).tolist(), [], 0
    for n in _lengths(case)[0]:
        paths = []
        for i in range(n):
            up = parent[r + i]
            paths.append((paths[up] if up >= 0 else []) + [i])
        out.append(paths)
        r += n
    return out


def _exact_tree(case, st, seed):
    words, mask, pos = _words(case), [], []
    for old, paths in zip(_lengths(case)[1], _paths(case, seed)):
        for p in paths:
            bits = sum(1 << i for i in p)
            for w in range(words):
                x = bits >> (64 * w) & (1 << 64) - 1
                mask.append(x - (1 << 64) if x >> 63 else x)
            pos.append(old + len(p) - 1)
    return {"mask": torch.tensor(mask, dtype=torch.int64, device="cuda").view(-1, words),
            "pos": torch.tensor(pos, dtype=torch.int32, device="cuda")}


def _exact_attend(case, st, seed):
    """Sequence by sequence and kv head by kv head."""
    nq, nkv, hd = _HEADS[case["model"]]
    rep = nq // nkv
    kc, vc, ks, vs = st["cache"]
    new, old = _lengths(case)
    out = torch.empty(sum(new), nq, hd, dtype=torch.float64, device="cuda")
    r = 0
    for s, (a, b, paths) in enumerate(zip(new, old, _paths(case, seed))):
        n = a + b
        ids = st["tab"][s, :(n + case["page"] - 1) // case["page"]].long()
        hidden = torch.ones(a, n, dtype=torch.bool)
        hidden[:, :b] = False
        for i, p in enumerate(paths):
            hidden[i, [b + x for x in p]] = False
        hidden = hidden.cuda()
        for h in range(nkv):
            k = kc[:, h].view(torch.uint8)[ids].view(kc.dtype).double() * ks[ids, h].double()[:, :, None]
            v = vc[:, h].view(torch.uint8)[ids].view(vc.dtype).double() * vs[ids, h].double()[:, :, None]
            k = k.view(-1, hd // 16, 16, 16).permute(0, 2, 1, 3).reshape(-1, hd)[:n]
            v = v.view(-1, 4, hd, 4).permute(0, 1, 3, 2).reshape(-1, hd)[:n]
            for i in range(h * rep, (h + 1) * rep):
                sc = (st["q"][r:r + a, i].double() @ k.T / math.sqrt(hd)).masked_fill_(hidden, -math.inf)
                out[r:r + a, i] = torch.softmax(sc, -1) @ v
        r += a
    return {"out": out}


def _nearest_code(x):
    """The e4m3 value nearest to x (ties to the even one), |x| <= 448, from the list of all of them."""
    all_ = [0.0] + [2.0 ** -9 * i for i in range(1, 8)] + [2.0 ** (e - 7) * (1 + f / 8) for e in range(1, 16) for f in range(8)]
    grid = torch.tensor(all_[:127], dtype=torch.float64, device="cuda")        # the last one's code is NaN
    a = x.abs()
    hi = torch.searchsorted(grid, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - a, a - grid[lo]
    pick = torch.where(up < down, hi, torch.where(up > down, lo, torch.where(hi % 2 == 0, hi, lo)))
    return torch.copysign(grid[pick], x)


def _exact_accept(case, st, seed):
    """Block by block in the sequences' own order, on values in 64 bits."""
    _, nkv, hd = _HEADS[case["model"]]
    m, pt = case["page"] // 16, case["page"]
    new, old = _lengths(case)
    kc, vc, ks, vs = st["cache"]
    pool = kc.shape[0]
    tab, last = st["tab"].cpu().tolist(), st["last"].cpu().tolist()
    length, blocks, sources = [], [], []                             # (page, sub) of blocks, and 16 flat places in the pool each
    for s, (a, b, paths) in enumerate(zip(new, old, _paths(case, seed))):
        keep = paths[last[s]] if last[s] >= 0 else []
        length.append(b + len(keep))
        place = lambda x: (tab[s][x // pt] * m + x % pt // 16) * 16 + x % 16  # noqa: E731
        for blk in range(b // 16, (b + len(keep) + 15) // 16):
            src = [t if t < b else b + keep[t - b] if t < b + len(keep) else None for t in range(16 * blk, 16 * blk + 16)]
            if any(x is not None and x != 16 * blk + i for i, x in enumerate(src)):
                blocks.append(place(16 * blk) // 16)
                sources.append([-1 if x is None else place(x) for x in src])
    got = {}
    for name, codes, scale in (("k", kc, ks), ("v", vc, vs)):
        shape = (pool, nkv, m, hd // 16, 16, 16) if name == "k" else (pool, nkv, m, 4, hd, 4)
        logical = codes.view(shape).double()                        # -> [pool * m * 16 tokens, nkv, dims]
        logical = (logical.transpose(3, 4) if name == "k" else logical.transpose(4, 5)).reshape(pool, nkv, m, 16, hd)
        logical = logical.permute(0, 2, 3, 1, 4).reshape(-1, nkv, hd).clone()
        factor = scale.double().permute(0, 2, 1).reshape(-1, nkv).clone()
        if blocks:
            dst, src = torch.tensor(blocks, device="cuda"), torch.tensor(sources, device="cuda")
            there, src = src >= 0, src.clamp(min=0)
            f = torch.where(there[..., None], factor[src // 16], torch.zeros((), dtype=torch.float64, device="cuda"))
            big = f.amax(1)                                          # [blocks, nkv]
            x = _nearest_code(logical[src] * (f / big[:, None])[..., None])
            flat = dst[:, None] * 16 + torch.arange(16, device="cuda")
            logical[flat[there]] = x[there]
            factor[dst] = big
        back = logical.view(pool, m, 16, nkv, hd).permute(0, 3, 1, 2, 4)
        back = back.reshape(pool, nkv, m, 16, hd // 16, 16).transpose(3, 4) if name == "k" else \
            back.reshape(pool, nkv, m, 4, 4, hd).transpose(4, 5)
        got[name] = back.reshape(codes.shape)
        got[name + "_scale"] = factor.view(pool, m, nkv).permute(0, 2, 1)
    return {**got, "len": torch.tensor(length, dtype=torch.int32, device="cuda")}


def _exact_sample(case, st, seed):
    """Row by row: logarithms of shares, the kept tokens as a list."""
    o, rows = st["opts"], case["rows"]
    at = lambda n: o[n].double().cpu().tolist() if isinstance(o[n], torch.Tensor) else [float(o[n])] * rows  # noqa: E731
    token, logprob, kept = [], [], []
    for r, (t, k, p, least, u) in enumerate(zip(at("temperature"), at("top_k"), at("top_p"), at("min_p"), st["u"].double().cpu().tolist())):
        z = st["z"][r].double()
        share = torch.log_softmax(z / t, 0)
        # by z, then by id: the key's second part never reaches the next z
        ids = torch.argsort(-z, stable=True)
        if k > 0:
            ids = ids[:int(k)]
        part = torch.softmax(z[ids] / t, 0)
        n = ids.numel()
        if p < 1:
            before = torch.cat([part.new_zeros(1), part.cumsum(0)[:-1]])
            n = int((before < p).sum())
        if least > 0:
            n = min(n, int((z[ids] >= z.max() + t * math.log(least)).sum()))
        ids = ids[:n].sort().values
        part = torch.log_softmax(z[ids] / t, 0)
        i = min(int(torch.searchsorted(part.exp().cumsum(0), torch.tensor([u], dtype=torch.float64, device="cuda"), right=True)), n - 1)
        token.append(ids[i])
        logprob.append(share[ids[i]])
        kept.append(part[i])
    return {"token": torch.stack(token).int(), "logprob": torch.stack(logprob), "kept": torch.stack(kept)}
