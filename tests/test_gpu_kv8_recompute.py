"""Recomputed log-probabilities of an 8-bit policy do not depend on how many other
sequences the call has: which pass the attention takes goes by the sequences that
have rows."""
import numpy as np
import pytest

from rg_helpers import prompts_to_device
from workload import ModelShape, make_weights

pytestmark = pytest.mark.gpu

GQA = ModelShape(2, 256, 12, 2, 128, 512, 2048, 1e6, dtype="bf16")


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


@pytest.mark.parametrize("at", [[0, 1], [500, 501], [1100, 1101], [3, 700]])
def test_sequences_without_rows_do_not_change_the_others(torch, at):
    """Two long completions alone and among 1100 of one token, whose only log-probability is the prompt's: the same rows
    go through the same products, and through the same attention as long as the empty ones do not count.  The
    log-probabilities are then the same bits; the row-by-row pass sums in another order and gives others."""
    import paper_2606_02218_amd as rg
    w = make_weights(GQA, 11)
    N, max_new = 1102, 90
    prompts = prompts_to_device([np.arange(1, 40, dtype=np.int32)])
    pol = rg.Policy(GQA, w, max_seqs=N, max_prompts=1, max_prompt_tokens=64, max_context=39 + max_new, kv_dtype="e4m3")
    rng = np.random.default_rng(2)
    two = torch.from_numpy(rng.integers(0, 2047, size=(2, max_new)).astype(np.int32)).cuda()
    n2 = torch.tensor([90, 71], dtype=torch.int32, device="cuda")
    alone = pol.recompute_logprobs(prompts, [2], two, n2)
    by_row = pol.recompute_logprobs(prompts, [2], two, n2, row_tiles=False)
    assert not torch.equal(alone, by_row)
    many = torch.from_numpy(rng.integers(0, 2047, size=(N, max_new)).astype(np.int32)).cuda()
    n = torch.ones(N, dtype=torch.int32, device="cuda")
    many[at], n[at] = two, n2
    got = pol.recompute_logprobs(prompts, [N], many, n)
    assert torch.equal(got[at], alone)
    assert torch.equal(pol.recompute_logprobs(prompts, [N], many, n, row_tiles=False)[at], by_row)
    got[at] = 0
    assert torch.all(got[:, 1:] == 0)
