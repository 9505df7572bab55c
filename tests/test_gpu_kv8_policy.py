"""Policies whose KV pool is in 8 bits: rollouts and recomputed log-probabilities
against the float64 decoder with the same cache, sharing, row tiles, chunks,
graphs, memory and refusals.

Tolerances.  The library's keys and values differ from the oracle's by the
rounding of its activations (17 bits and fp32 sums); where one lies next to a
border of the codes it takes the other, a step of up to 2^-3 of it.  What that
may do is measured on the oracle alone: the change of its log-probabilities when
keys and values get relative noise of 2^-14, eight times the activations' 2^-17.
Four times that change (its maximum and its mean square) bounds the library's.
"""
import numpy as np
import pytest

from oracle.grpo import teacher_forced_logprobs
from oracle.kv8 import Kv8Model
from oracle.rollout import rollout as oracle_rollout
from rg_helpers import oracle_for, prompts_to_device
from workload import ModelShape, make_weights

pytestmark = pytest.mark.gpu

GQA = ModelShape(2, 256, 12, 2, 128, 512, 2048, 1e6, dtype="bf16")
MHA = ModelShape(2, 768, 12, 12, 64, 1024, 2048, 1e4, dtype="bf16")


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


def _policy(shape, w, prompts, G, max_new, kv="e4m3", **kw):
    import paper_2606_02218_amd as rg
    lim = dict(max_seqs=int(np.sum(G)), max_prompts=len(G), max_prompt_tokens=int(sum(map(len, prompts))),
               max_context=max(map(len, prompts)) + max_new)
    return rg.Policy(shape, w, kv_dtype=kv, **{**lim, **kw})


def _case(shape, plens, G, max_new, seed):
    rng = np.random.default_rng(seed)
    prompts = [rng.integers(0, shape.vocab - 1, size=n).astype(np.int32) for n in plens]
    L = rng.integers(2, max_new + 1, size=int(np.sum(G))).astype(np.int32)
    L[0], L[-1] = 1, max_new
    return prompts, L


def _valid(lengths, max_new):
    return np.arange(max_new)[None] < np.asarray(lengths)[:, None]


def _noise(shape, w, prompts, G, ref, max_new):
    """(log-probabilities of the oracle, largest and mean square change under noise)."""
    want = teacher_forced_logprobs(Kv8Model(shape, w), prompts, G, ref["tokens"], ref["lengths"])
    v = _valid(ref["lengths"], max_new)
    d = np.stack([teacher_forced_logprobs(Kv8Model(shape, w, jitter=2.0 ** -14, seed=s), prompts, G, ref["tokens"],
                                          ref["lengths"]) - want for s in (1, 2)])[:, v]
    return want, np.abs(d).max(), np.sqrt((d ** 2).mean())


CASES = [(GQA, (37, 16, 5), [3, 2, 4], 40), (MHA, (33, 15, 17, 48), [2, 1, 3, 2], 30), (GQA, (300,), [2], 20)]


@pytest.mark.parametrize("shape,plens,G,max_new", CASES)
def test_rollout_and_recompute_against_the_oracle(torch, shape, plens, G, max_new):
    w = make_weights(shape, 3)
    prompts, L = _case(shape, plens, G, max_new, 5)
    ref = oracle_rollout(Kv8Model(shape, w), prompts, G, max_new, 1, L)
    want, top, rms = _noise(shape, w, prompts, G, ref, max_new)
    plain = teacher_forced_logprobs(oracle_for(shape, w), prompts, G, ref["tokens"], ref["lengths"])
    v = _valid(ref["lengths"], max_new)
    assert np.sqrt(((plain - want)[v] ** 2).mean()) > 6 * rms      # well over the bound below: the cache's own rounding shows
    pol = _policy(shape, w, prompts, G, max_new)
    dp = prompts_to_device(prompts)
    force = torch.from_numpy(ref["tokens"]).cuda()
    _, ln, lp = pol.rollout(dp, G, max_new, 1, forced_len=L, force_tokens=force)
    assert np.array_equal(ln.cpu().numpy(), ref["lengths"])
    lp = lp.cpu().numpy()
    for got in (lp, pol.recompute_logprobs(dp, G, force, ln).cpu().numpy(),
                pol.recompute_logprobs(dp, G, force, ln, row_tiles=False).cpu().numpy()):
        err = (got - want)[v]
        print(f"max {np.abs(err).max():.2e} of {4 * top:.2e}, rms {np.sqrt((err ** 2).mean()):.2e} of {4 * rms:.2e}", flush=True)
        assert np.abs(err).max() <= 4 * top and np.sqrt((err ** 2).mean()) <= 4 * rms
        assert np.all(got[~v] == 0)


def test_private_pages_graphs_and_profiling_change_nothing(torch):
    w = make_weights(GQA, 4)
    prompts, L = _case(GQA, (50, 16, 31), [4, 3, 2], 24, 6)
    G = [4, 3, 2]
    pol = _policy(GQA, w, prompts, G, 24)
    dp = prompts_to_device(prompts)
    a = pol.rollout(dp, G, 24, 9, forced_len=L)
    for kw in (dict(share_prefix=False), dict(profile=True), dict(group_prefix_pass=True)):
        b = pol.rollout(dp, G, 24, 9, forced_len=L, **kw)
        assert all(torch.equal(x, y) for x, y in zip(a, b)), kw
        if "profile" in kw:
            times = pol.kernel_times(1)
            assert times["qkv_rope"][1] > 0 and times["attn"][1] > 0
    r = pol.recompute_logprobs(dp, G, a[0], a[1])
    assert torch.equal(r, pol.recompute_logprobs(dp, G, a[0], a[1], share_prefix=False))


def test_long_contexts_are_split(torch):
    """Few rows of a long prompt: the decode attention is cut into chunks; the recompute's rows pass too."""
    w = make_weights(GQA, 5)
    prompts, G, max_new = [np.random.default_rng(1).integers(0, 2047, size=2100).astype(np.int32)], [2], 6
    L = np.array([6, 4], np.int32)
    ref = oracle_rollout(Kv8Model(GQA, w), prompts, G, max_new, 1, L)
    want, top, rms = _noise(GQA, w, prompts, G, ref, max_new)
    pol = _policy(GQA, w, prompts, G, max_new)
    dp, force = prompts_to_device(prompts), torch.from_numpy(ref["tokens"]).cuda()
    _, ln, lp = pol.rollout(dp, G, max_new, 1, forced_len=L, force_tokens=force)
    v = _valid(L, max_new)
    for got in (lp, pol.recompute_logprobs(dp, G, force, ln), pol.recompute_logprobs(dp, G, force, ln, row_tiles=False)):
        err = (got.cpu().numpy() - want)[v]
        assert np.abs(err).max() <= 4 * top and np.sqrt((err ** 2).mean()) <= 4 * rms, (np.abs(err).max(), top)


def test_recompute_in_chunks(torch):
    """More completion rows than a chunk holds: a chunk ends inside a sequence and inside a block, and the next one
    goes on there, as a decode does."""
    w = make_weights(GQA, 6)
    prompts, G, max_new = [np.arange(1, 20, dtype=np.int32), np.arange(5, 12, dtype=np.int32)], [24, 24], 110
    rng = np.random.default_rng(3)
    tok = torch.from_numpy(rng.integers(0, 2047, size=(48, max_new)).astype(np.int32)).cuda()
    ln = torch.from_numpy(rng.integers(70, max_new + 1, size=48).astype(np.int32)).cuda()
    pol = _policy(GQA, w, prompts, G, max_new)
    assert int(ln.sum()) - 48 > 4096                              # a chunk's most rows
    dp = prompts_to_device(prompts)
    whole = pol.recompute_logprobs(dp, G, tok, ln).cpu().numpy()
    # each sequence alone: one chunk
    solo = _policy(GQA, w, prompts, [1, 1], max_new)
    sub = [3, 30, 45]
    t, n = tok.cpu().numpy(), ln.cpu().numpy()
    for s in sub:
        p = s // 24
        one = solo.recompute_logprobs([dp[p]], [1], tok[s:s + 1].contiguous(), ln[s:s + 1].contiguous()).cpu().numpy()[0]
        ref = dict(tokens=t[s:s + 1], lengths=n[s:s + 1])
        want, top, rms = _noise(GQA, w, [prompts[p]], [1], ref, max_new)
        v = _valid(n[s:s + 1], max_new)[0]
        for got in (one, whole[s]):
            err = (got - want[0])[v]
            assert np.abs(err).max() <= 4 * top and np.sqrt((err ** 2).mean()) <= 4 * rms


def test_many_sequences_that_retire(torch):
    """Decode steps of rows enough to be taken by length, fewer with every step: sequences against the oracle's alone."""
    w = make_weights(MHA, 7)
    prompts, G, max_new = [np.arange(1, 40, dtype=np.int32), np.arange(5, 12, dtype=np.int32)], [50, 45], 40
    rng = np.random.default_rng(4)
    t = rng.integers(0, 2047, size=(95, max_new)).astype(np.int32)
    n = rng.integers(1, max_new + 1, size=95).astype(np.int32)
    n[[0, 60]], n[[22, 49, 94]] = max_new, (25, 31, 28)
    t[np.arange(95), n - 1] = 2047                                # the last token of a sequence is the end
    t[~_valid(n, max_new)] = -1
    pol = _policy(MHA, w, prompts, G, max_new)
    dp, force = prompts_to_device(prompts), torch.from_numpy(t).cuda()
    _, ln, lp = pol.rollout(dp, G, max_new, 1, forced_len=n, force_tokens=force)
    assert np.array_equal(ln.cpu().numpy(), n)
    lp, by_rows = lp.cpu().numpy(), pol.recompute_logprobs(dp, G, force, ln, row_tiles=False).cpu().numpy()
    for s in (0, 22, 49, 60, 94):
        p = int(s >= 50)
        ref = dict(tokens=t[s:s + 1], lengths=n[s:s + 1])
        want, top, rms = _noise(MHA, w, [prompts[p]], [1], ref, max_new)
        v = _valid(n[s:s + 1], max_new)[0]
        for got in (lp[s], by_rows[s]):
            err = (got - want[0])[v]
            assert np.abs(err).max() <= 4 * top, (s, np.abs(err).max(), top)


def test_memory_and_refusals(torch):
    import paper_2606_02218_amd as rg
    w = make_weights(GQA, 4)
    prompts = [np.arange(1, 33, dtype=np.int32)]
    big = dict(kv_pool_pages=40000)
    a = _policy(GQA, w, prompts, [2], 16, kv=None, **big)
    b = _policy(GQA, w, prompts, [2], 16, **big)
    pool = 2 * 40000 * 2 * 2 * 16 * 128 * 2                       # layers, pages, k and v, heads, tokens, dims, bytes
    scales = 2 * 40000 * 2 * 2 * 4
    assert a.device_bytes() - b.device_bytes() >= pool // 2 - scales - (16 << 20)
    with pytest.raises(ValueError, match="kv_dtype"):
        _policy(GQA, w, prompts, [2], 16, kv="int8")
    tiny = ModelShape(1, 64, 2, 2, 32, 128, 64, 1e4, dtype="f32")
    with pytest.raises(rg.RolloutError, match="bf16 model"):
        _policy(tiny, make_weights(tiny, 0), [np.arange(1, 5, dtype=np.int32)], [1], 4)
    with pytest.raises(rg.RolloutError, match="ran out"):
        p = _policy(GQA, w, prompts, [2], 64, kv_pool_pages=4)
        p.rollout(prompts_to_device(prompts), [2], 64, 0, forced_len=[64, 64])
