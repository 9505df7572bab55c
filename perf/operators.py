"""Rotary positions and an 8-bit paged key/value cache: their calls as cases to
be timed and checked.

Three operators: ``rope`` (rotary positions and their gradient), ``kv8_append``
(rotate, quantize and append keys and values, queries rotated on the way) and
``kv8_attention`` (causal attention over that cache, one row a sequence or
ragged runs of rows).  ``run`` computes each in elementary torch operations,
or, with ``own`` set, by the library's entry points.

The cache.  16 consecutive tokens of one kv head are a block with one scale, a
power of two; a page is page_tokens / 16 blocks of every kv head, a sequence a
row of page ids.  A value is an e4m3 code times its block's scale.  Inside a
block, keys lie as [dim / 16][token][dim % 16], values as
[token / 4][dim][token % 4].

Append.  A block's scale is 2^k for the least k in [-64, 119] with 448 * 2^k >=
the largest magnitude among its new rows, or its old scale where tokens before
them stay in the block and that is larger.  Codes round to nearest even; tokens
that stay are requantized where the scale grows.
"""
import math
import random

import torch

own = False

# (query heads, kv heads, head_dim) of the repository's bf16 workloads
_HEADS = {"gpt2s": (12, 12, 64), "1.5b": (12, 2, 128), "7b": (28, 4, 128)}
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rope(rows, heads, hd, rot, layout, dtype, scaling="none", inverse=False, max_pos=4608, name=None):
    c = {"name": name} if name else {}
    c.update(kind="rope", rows=rows, heads=heads, head_dim=hd, rot=rot, layout=layout, dtype=dtype, scaling=scaling,
             inverse=inverse, max_pos=max_pos)
    return c


def _append(model, seqs, new, old, dtype, rot=0, layout="half", scaling="none", page=16, name=None):
    """new, old: (lo, hi) rows that a sequence appends and tokens that it holds already; rot 0: the whole head."""
    c = {"name": name} if name else {}
    c.update(kind="append", model=model, seqs=seqs, new_lo=new[0], new_hi=new[1], old_lo=old[0], old_hi=old[1],
             dtype=dtype, rot=rot or _HEADS[model][2], layout=layout, scaling=scaling, page=page)
    return c


def _attend(model, seqs, new, old, dtype, group=1, shared=0, page=16, name=None):
    """As _append; every `group` sequences share the pages of their first `shared` tokens."""
    c = {"name": name} if name else {}
    c.update(kind="attend", model=model, seqs=seqs, new_lo=new[0], new_hi=new[1], old_lo=old[0], old_hi=old[1],
             dtype=dtype, group=group, shared=shared, page=page)
    return c


def listed():
    return [
        # One decode step's queries for a handful of sequences: latency only.
        _rope(8, 12, 64, 64, "half", "bf16", name="rope_step_8"),
        # The queries of a full batch's prompts (32 x 512 tokens) at the larger decoder's widths.
        _rope(16384, 28, 128, 128, "half", "bf16", name="rope_prompts_7b"),
        # The gradient at the queries of an odd number of rows: interleaved pairs, the first half of each head, fp32,
        # positions past the trained length with frequencies scaled by bands.
        _rope(7001, 12, 128, 64, "interleaved", "f32", scaling="bands", inverse=True, max_pos=32768,
              name="rope_grad_part_long"),
        # The straggler tail of a rollout: the few sequences left append one token each.
        _append("1.5b", 8, (1, 1), (900, 4500), "bf16", name="append_tail_1.5b"),
        # A decode step of the full training batch, 32 prompts x 16.
        _append("1.5b", 512, (1, 1), (512, 2600), "bf16", name="append_step_1.5b"),
        # The prefill of the full batch: 32 prompts of 512 tokens into empty pages, at the larger decoder's widths.
        _append("7b", 32, (512, 512), (0, 0), "bf16", name="append_prompts_7b"),
        # Odd chunks behind odd histories (a turn's new tokens), fp32 projections, interleaved pairs on half the head.
        _append("gpt2s", 37, (3, 211), (0, 700), "f32", rot=32, layout="interleaved", scaling="linear", page=64,
                name="append_chunks_gpt2s"),
        # A few sequences of the small model: latency.
        _attend("gpt2s", 8, (1, 1), (200, 600), "bf16", name="attend_step_gpt2s"),
        # A decode step of the full training batch: 512 rows, prompts' pages shared by groups of 16.
        _attend("1.5b", 512, (1, 1), (512, 2600), "bf16", group=16, shared=512, name="attend_step_1.5b"),
        # A few very long sequences: the work of each has to be split.
        _attend("7b", 3, (1, 1), (60001, 131000), "bf16", page=64, name="attend_long_7b"),
        # A rollout's recompute in the fp32 activations of the policies: odd runs behind shared prompts.
        _attend("1.5b", 24, (37, 701), (131, 131), "f32", group=8, shared=128, name="attend_runs_1.5b"),
        # Prompts in chunks: 2048 rows each behind what the cache holds already, bound by the products.
        _attend("7b", 4, (2048, 2048), (2000, 6144), "bf16", name="attend_chunk_7b"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: sizes log-uniform, odd ones among them."""
    dtype = rng.choice(["bf16", "bf16", "f32"])
    layout, scaling = rng.choice(["half", "half", "interleaved"]), rng.choice(["none", "none", "linear", "base", "bands"])
    kind = rng.choice(["rope", "append step", "append run", "attend step", "attend long", "attend run"])
    model = rng.choice(sorted(_HEADS))
    nq, nkv, hd = _HEADS[model]
    rot = hd if rng.random() < 0.6 else 2 * rng.randint(hd // 8, hd // 2)
    page = rng.choice([16, 16, 32, 64])
    if kind == "rope":
        return _rope(_log_int(rng, 1, 8000), rng.choice([nq, nkv, rng.randint(1, 28)]), hd, rot, layout, dtype, scaling,
                     rng.random() < 0.5, _log_int(rng, 64, 32768))
    lo = _log_int(rng, 1, 2600)
    if kind == "append step":
        return _append(model, _log_int(rng, 1, 512), (1, 1), (rng.choice([0, lo]), lo + rng.randint(0, 900)), dtype, rot,
                       layout, scaling, page)
    if kind == "append run":
        n = _log_int(rng, 2, 400)
        return _append(model, _log_int(rng, 1, 24), (1, n), (0, rng.randint(0, 900)), dtype, rot, layout, scaling, page)
    if kind == "attend step":
        g = rng.choice([1, 1, 4, 16])
        return _attend(model, g * _log_int(rng, 1, 320 // g), (1, 1), (lo, lo + rng.randint(0, 1200)), dtype, g,
                       16 * rng.randint(0, lo // 16) if g > 1 and page == 16 else 0, page)
    if kind == "attend long":
        n = _log_int(rng, 4000, 100000)
        return _attend(model, rng.randint(1, 4), (1, rng.choice([1, 1, 2, 5])), (n, n + rng.randint(0, n // 4)), dtype,
                       page=page)
    n = _log_int(rng, 2, 700)
    return _attend(model, _log_int(rng, 1, 16), (1, n), (0, _log_int(rng, 16, 2000)), dtype, page=page)


# ---------------------------------------------------------------- inputs
def _theta(case):
    return 1e6 if case["kind"] == "rope" or _HEADS[case["model"]][2] == 128 else 1e4


#: (factor, trained length, slow turns, fast turns) of scaled frequencies
_SCALE = (4.0, 4096, 1.0, 32.0)


def _frequencies(case):
    """The angles per position of each pair, in 64 bits, and the amplitude."""
    rot, theta = case["rot"], _theta(case)
    f, length, slow, fast = _SCALE
    i = torch.arange(rot // 2, device="cuda", dtype=torch.float64)
    if case["scaling"] == "base":
        theta = theta * f ** (rot / (rot - 2))
    w = theta ** (-2.0 * i / rot)
    if case["scaling"] == "linear":
        w = w / f
    if case["scaling"] == "bands":
        keep = ((w * length / (2 * math.pi) - slow) / (fast - slow)).clamp(0.0, 1.0)
        return w * (keep + (1.0 - keep) / f), 0.1 * math.log(f) + 1.0
    return w, 1.0


def _table(case, n):
    """cos and sin of positions below n: fp32 [n, rot / 2], as a program makes them once."""
    w, amp = _frequencies(case)
    a = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * w
    return (amp * a.cos()).float(), (amp * a.sin()).float()


def _lengths(case):
    """(new rows, tokens held before them) of every sequence; they follow from the case alone."""
    r = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]
    return new, [r.randint(case["old_lo"], case["old_hi"]) for _ in range(case["seqs"])]


def _pages(case, gen):
    """A page table of scattered pages (the sequences of a group share the pages of their first `shared` tokens) and
    the number of pages of the pool."""
    new, old = _lengths(case)
    pt = case["page"]
    width = max((a + b + pt - 1) // pt for a, b in zip(new, old))
    S, g, sh = case["seqs"], case.get("group", 1), case.get("shared", 0) // pt
    need = torch.tensor([(a + b + pt - 1) // pt for a, b in zip(new, old)], device="cuda")
    at = torch.arange(width, device="cuda")[None].expand(S, width)
    ids = torch.arange(S * width, device="cuda").view(S, width)
    first = torch.arange(S, device="cuda")[:, None] // g * g * width + at
    ids = torch.where(at < sh, first, ids)
    used, dense = torch.unique(ids[at < need[:, None]], return_inverse=True)
    pool = used.numel() + 3                                         # a pool holds pages of nobody too
    perm = torch.randperm(pool, generator=gen, device="cuda")
    tab = torch.zeros(S, width, dtype=torch.int64, device="cuda")
    tab[at < need[:, None]] = perm[dense]
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


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 11)
    dt = _DT[case["dtype"]]
    if case["kind"] == "rope":
        x = torch.randn(case["rows"], case["heads"], case["head_dim"], generator=gen, device="cuda").to(dt)
        pos = torch.randint(0, case["max_pos"], (case["rows"],), generator=gen, device="cuda", dtype=torch.int32)
        cos, sin = _table(case, case["max_pos"])
        return {"case": case, "x": x, "pos": pos, "cos": cos, "sin": sin}
    new, old = _lengths(case)
    nq, nkv, hd = _HEADS[case["model"]]
    rows = sum(new)
    tab, pool = _pages(case, gen)
    st = {"case": case, "tab": tab, "cache": _pool(case, pool, gen), "max_len": max(a + b for a, b in zip(new, old)),
          "max_new": max(new), "len": torch.tensor([a + b for a, b in zip(new, old)], device="cuda", dtype=torch.int32)}
    # a step's rows need no offsets: row s is sequence s
    st["off"] = None if case["new_hi"] == 1 else torch.tensor([0] + new, device="cuda").cumsum(0).int()
    if case["kind"] == "append":
        # one projection's output [rows, q | k | v]; its channels differ in size
        gain = torch.exp(0.6 * torch.randn((nq + 2 * nkv) * hd, generator=gen, device="cuda"))
        qkv = (torch.randn(rows, (nq + 2 * nkv) * hd, generator=gen, device="cuda") * gain).to(dt)
        cut = qkv.view(rows, nq + 2 * nkv, hd)
        st["q"], st["k"], st["v"] = cut[:, :nq], cut[:, nq:nq + nkv], cut[:, nq + nkv:]
        st["cos"], st["sin"] = _table(case, st["max_len"])
    else:
        st["q"] = (1.5 * torch.randn(rows, nq, hd, generator=gen, device="cuda")).to(dt)
    return st


# ---------------------------------------------------------------- the plain form
def _rotate(x, cos, sin, rot, layout):
    """x [rows, heads, hd] with each row's cos and sin [rows, rot / 2], in their type."""
    x, c, s = x.to(cos.dtype), cos[:, None], sin[:, None]
    m = rot // 2
    if layout == "half":
        a, b = x[..., :m], x[..., m:rot]
        return torch.cat([a * c - b * s, b * c + a * s, x[..., rot:]], -1)
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), x[..., rot:]], -1)


def _row_places(state):
    """The sequence of every row and its position there."""
    n, off = state["len"].long(), state["off"]
    if off is None:
        return torch.arange(n.numel(), device="cuda"), n - 1
    rows = torch.arange(state["q"].shape[0], device="cuda")
    seq = torch.bucketize(rows, off[1:].long(), right=True)
    return seq, n[seq] - (off[seq + 1].long() - rows)


def _power(amax):
    """The block scale 2^k of a largest magnitude."""
    m, e = torch.frexp(amax)
    k = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.exp2(torch.where(amax > 0, k, -64).clamp(-64, 119).double())


def _plain_append(state):
    case = state["case"]
    nq, nkv, hd = _HEADS[case["model"]]
    m, pt = case["page"] // 16, case["page"]
    seq, pos = _row_places(state)
    cos, sin = state["cos"][pos], state["sin"][pos]
    q = _rotate(state["q"], cos, sin, case["rot"], case["layout"]).to(state["q"].dtype)
    # 64 bits: a code depends on which side of a border its value lies
    k = _rotate(state["k"], cos.double(), sin.double(), case["rot"], case["layout"])
    v = state["v"].double()
    tab = state["tab"].long()
    block = tab[seq, pos // pt] * m + pos % pt // 16                 # of each row, over the whole pool
    start = state["len"].long()
    start = start - (1 if state["off"] is None else (state["off"][1:] - state["off"][:-1]).long())
    held = start % 16 != 0                                           # sequences whose first block holds older tokens
    at = start.clamp(max=tab.shape[1] * pt - 1)
    fore = (tab.gather(1, (at // pt)[:, None])[:, 0] * m + at % pt // 16)[held]
    keep = torch.arange(16, device="cuda") < (start % 16)[held][:, None]   # [blocks, 16]
    slot, head = pos % 16, torch.arange(nkv, device="cuda")
    for_k, for_v = state["cache"][:2], state["cache"][2:]
    for x, codes, scale, keys in ((k, for_k[0], for_v[0], True), (v, for_k[1], for_v[1], False)):
        pool = codes.shape[0]
        view = codes.view(pool, nkv, m, hd // 16, 16, 16) if keys else codes.view(pool, nkv, m, 4, hd, 4)
        amax = torch.zeros(pool * m, nkv, dtype=torch.float64, device="cuda")
        amax.scatter_reduce_(0, block[:, None].expand(-1, nkv), x.abs().amax(-1), "amax")
        flat = scale.transpose(1, 2).reshape(pool * m, nkv).double()
        grown = _power(amax)
        grown[fore] = torch.maximum(grown[fore], flat[fore])
        touched = torch.zeros(pool * m, dtype=torch.bool, device="cuda")
        touched[block] = True
        grown = torch.where(touched[:, None], grown, flat)
        # tokens that stay: requantized by the growth
        page, sub = fore // m, fore % m
        was = view.view(torch.uint8)[page, :, sub].view(codes.dtype).double()
        keepers = (keep[:, None, None, :, None] if keys else keep.view(-1, 1, 4, 1, 4)).expand(was.shape)
        ratio = (flat[fore] / grown[fore])[:, :, None, None, None]
        again = torch.where(keepers, was * ratio, was).float().to(codes.dtype)
        view.view(torch.uint8)[page, :, sub] = again.view(torch.uint8)
        new = (x / grown[block][:, :, None]).float().to(codes.dtype).view(torch.uint8)
        page, sub = (block // m)[:, None], (block % m)[:, None]
        if keys:
            view.view(torch.uint8)[page, head[None], sub, :, slot[:, None]] = new.view(-1, nkv, hd // 16, 16)
        else:
            view.view(torch.uint8)[page, head[None], sub, slot[:, None] // 4, :, slot[:, None] % 4] = new
        scale.copy_(grown.float().view(pool, m, nkv).transpose(1, 2))
    kc, vc, ks, vs = state["cache"]
    return {"q": q, "k": kc, "v": vc, "k_scale": ks, "v_scale": vs}


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
    seq, pos = _row_places(state)
    S, L, R = case["seqs"], state["max_len"], state["max_new"]
    tab = state["tab"].long()
    k = _gathered(kc, ks, tab, hd, True)[:, :, :L]
    row = torch.zeros_like(seq) if state["off"] is None else torch.arange(seq.numel(), device="cuda") - state["off"].long()[seq]
    q = torch.zeros(S, R, nkv, rep, hd, device="cuda")
    q[seq, row] = state["q"].float().view(-1, nkv, rep, hd)
    last = torch.full((S, R), -1, device="cuda")
    last[seq, row] = pos
    s = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(S, nkv, R * rep, hd), k.transpose(2, 3)).mul_(hd ** -0.5)
    del k
    seen = torch.arange(L, device="cuda") <= last[:, :, None]       # [S, R, L]
    s = s.view(S, nkv, R, rep, L).masked_fill_(~seen[:, None, :, None], -math.inf)
    s.sub_(s.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(S, nkv, R * rep, L), _gathered(vc, vs, tab, hd, False)[:, :, :L]).view(S, nkv, R, rep, hd)
    o = (o / total.clamp(min=1e-30)).permute(0, 2, 1, 3, 4).reshape(S, R, nq, hd)
    return {"out": o[seq, row].to(state["q"].dtype)}


def run(state):
    case = state["case"]
    if own:
        import paper_2606_02218_amd as rg
        if case["kind"] == "rope":
            return {"y": rg.rope(state["x"], state["pos"], state["cos"], state["sin"], layout=case["layout"],
                                 inverse=case["inverse"])}
        cache = rg.Kv8Cache(*state["cache"])
        if case["kind"] == "append":
            q = rg.kv8_append(cache, state["k"], state["v"], state["tab"], state["len"], state["off"], q=state["q"],
                              cos=state["cos"], sin=state["sin"], layout=case["layout"])
            return {"q": q, "k": cache.k, "v": cache.v, "k_scale": cache.k_scale, "v_scale": cache.v_scale}
        return {"out": rg.kv8_attention(cache, state["q"], state["tab"], state["len"], state["off"],
                                        max_len=state["max_len"])}
    if case["kind"] == "rope":
        pos = state["pos"].long()
        cos, sin = state["cos"][pos], state["sin"][pos]
        y = _rotate(state["x"], cos, -sin if case["inverse"] else sin, case["rot"], case["layout"])
        return {"y": y.to(state["x"].dtype)}
    return _plain_append(state) if case["kind"] == "append" else _plain_attend(state)


def work(case):
    eb = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "rope":
        n = case["rows"] * case["heads"] * case["head_dim"]
        return {"bytes": 2 * n * eb + case["rows"] * (4 + 4 * case["rot"]),
                "flops": 3 * case["rows"] * case["heads"] * case["rot"]}
    nq, nkv, hd = _HEADS[case["model"]]
    new, old = _lengths(case)
    rows = sum(new)
    if case["kind"] == "append":
        blocks = sum((a + b + 15) // 16 - b // 16 for a, b in zip(new, old))
        return {"bytes": rows * ((2 * nq + 2 * nkv) * hd * eb + 2 * nkv * hd + 4 * case["rot"]) + 16 * blocks * nkv,
                "flops": rows * (3 * (nq + nkv) * case["rot"] + 6 * nkv * hd)}
    pairs = sum(a * b + a * (a + 1) // 2 for a, b in zip(new, old))
    g, sh = case["group"], case["shared"] // case["page"] * case["page"]
    tokens = sum(a + b for a, b in zip(new, old)) - (case["seqs"] - (case["seqs"] + g - 1) // g) * sh
    return {"bytes": tokens * nkv * (2 * hd + 0.5) + 2 * rows * nq * hd * eb, "flops": 4 * hd * nq * pairs}


# ---------------------------------------------------------------- 64 bits
def exact(case, seed):
    with torch.no_grad():
        st = prepare(case, seed)
        if case["kind"] == "rope":
            y = _exact_rotation(case, st["x"], st["pos"], case["inverse"])
            return {"y": y}
        new, old = _lengths(case)
        if case["kind"] == "append":
            return _exact_append(case, st, new, old)
        return _exact_attend(case, st, new, old)


def _exact_rotation(case, x, pos, inverse=False):
    """Pairs as complex numbers, turned by the angle itself (no table)."""
    w, amp = _frequencies(case)
    rot = case["rot"]
    turn = torch.polar(torch.full_like(w, amp).expand(pos.numel(), -1), pos.double()[:, None] * w)[:, None]
    if inverse:
        turn = turn.conj()
    x = x.double().clone()
    if case["layout"] == "half":
        z = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * turn
        x[..., :rot // 2], x[..., rot // 2:rot] = z.real, z.imag
    else:
        z = torch.view_as_complex(x[..., :rot].reshape(*x.shape[:2], rot // 2, 2)) * turn
        x[..., :rot] = torch.view_as_real(z).flatten(-2)
    return x


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


def _exact_append(case, st, new, old):
    """Block by block in the sequences' own order, on values in 64 bits."""
    nq, nkv, hd = _HEADS[case["model"]]
    m, pt = case["page"] // 16, case["page"]
    pos = torch.cat([torch.arange(b, b + a, device="cuda") for a, b in zip(new, old)])
    q = _exact_rotation(case, st["q"], pos)
    xs = (_exact_rotation(case, st["k"], pos), st["v"].double())
    kc, vc, ks, vs = st["cache"]
    pool = kc.shape[0]
    tab = st["tab"].cpu().tolist()
    # every touched block: (page, part, first slot that is new), and its new rows among all
    place, first, rows = [], [], []
    r = 0
    for s, (a, b) in enumerate(zip(new, old)):
        p = b
        while p < a + b:
            n = min(16 - p % 16, a + b - p)
            place.append((tab[s][p // pt], p % pt // 16))
            first.append(p % 16)
            rows.append([r + i if i < n else -1 for i in range(16)])
            p, r = p + n, r + n
    pg, sub = (torch.tensor(x, device="cuda") for x in zip(*place))
    first, rows = torch.tensor(first, device="cuda"), torch.tensor(rows, device="cuda")
    got = {}
    t = torch.arange(16, device="cuda")
    for name, x, codes, scale in (("k", xs[0], kc, ks), ("v", xs[1], vc, vs)):
        shape = (pool, nkv, m, hd // 16, 16, 16) if name == "k" else (pool, nkv, m, 4, hd, 4)
        logical = codes.view(shape).double()                        # -> [pool, nkv, m, token, dim]
        logical = (logical.transpose(3, 4) if name == "k" else logical.transpose(4, 5)).reshape(pool, nkv, m, 16, hd).clone()
        held = logical[pg, :, sub]                                  # [blocks, nkv, 16, hd]
        src = (rows.gather(1, (t[None] - first[:, None]).clamp(min=0)))
        fresh = (t[None] >= first[:, None]) & (src >= 0)
        val = x[src.clamp(min=0)].transpose(1, 2)                   # [blocks, nkv, 16, hd]
        val = torch.where(fresh[:, None, :, None], val, torch.zeros_like(val))
        amax = val.abs().amax((2, 3))
        k = torch.ceil(torch.log2(amax / 448.0)).clamp(-64, 119).nan_to_num(neginf=-64)
        k = torch.where(torch.exp2(k) * 448.0 < amax, k + 1, k)
        k = torch.where((torch.exp2(k - 1) * 448.0 >= amax) & (k > -64), k - 1, k)
        s_old = scale[pg, :, sub].double()
        s_new = torch.exp2(k)
        s_new = torch.where((first > 0)[:, None], torch.maximum(s_new, s_old), s_new)
        stay = t[None] < first[:, None]
        held = torch.where(stay[:, None, :, None], _nearest_code(held * (s_old / s_new)[:, :, None, None]), held)
        held = torch.where(fresh[:, None, :, None], _nearest_code(val / s_new[:, :, None, None]), held)
        logical[pg, :, sub] = held
        back = logical.view(pool, nkv, m, 16, hd // 16, 16).transpose(3, 4) if name == "k" else \
            logical.view(pool, nkv, m, 4, 4, hd).transpose(4, 5)
        got[name] = back.reshape(codes.shape)
        got[name + "_scale"] = scale.double().clone()
        got[name + "_scale"][pg, :, sub] = s_new
    return {"q": q, **got}


def _exact_attend(case, st, new, old):
    """Sequence by sequence and kv head by kv head."""
    nq, nkv, hd = _HEADS[case["model"]]
    rep = nq // nkv
    kc, vc, ks, vs = st["cache"]
    out = torch.empty(sum(new), nq, hd, dtype=torch.float64, device="cuda")
    r = 0
    for s, (a, b) in enumerate(zip(new, old)):
        n = a + b
        ids = st["tab"][s, :(n + case["page"] - 1) // case["page"]].long()
        hidden = torch.arange(n, device="cuda")[None] > torch.arange(b, n, device="cuda")[:, None]
        for h in range(nkv):
            k = kc[:, h].view(torch.uint8)[ids].view(kc.dtype).double() * ks[ids, h].double()[:, :, None]
            v = vc[:, h].view(torch.uint8)[ids].view(vc.dtype).double() * vs[ids, h].double()[:, :, None]
            k = k.view(-1, hd // 16, 16, 16).permute(0, 2, 1, 3).reshape(-1, hd)[:n]
            v = v.view(-1, 4, hd, 4).permute(0, 1, 3, 2).reshape(-1, hd)[:n]
            for j in range(h * rep, (h + 1) * rep):
                sc = (st["q"][r:r + a, j].double() @ k.T / math.sqrt(hd)).masked_fill_(hidden, -math.inf)
                out[r:r + a, j] = torch.softmax(sc, -1) @ v
        r += a
    return {"out": out}
