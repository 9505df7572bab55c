"""The drafted-tree oracle against cases worked out by hand."""
import numpy as np
import pytest

from oracle import kv8, tree


def test_masks_of_a_small_tree():
    #        0        a chain 0-1-3 and a branch 0-2-4
    mask, pos = tree.masks([-1, 0, 0, 1, 2], 1, 10)
    assert mask[:, 0].tolist() == [0b1, 0b11, 0b101, 0b1011, 0b10101]
    assert pos.tolist() == [10, 11, 11, 12, 12]


def test_masks_of_forests_padding_and_wrong_parents():
    mask, pos = tree.masks([-1, -1, 1, 7, 3, -2], 1, 0)
    assert mask[:, 0].tolist() == [1, 2, 6, 0, 0, 0] and pos.tolist() == [0, 0, 1, -1, -1, -1]
    mask, pos = tree.masks([-1, 0, 1, 2], 1, 0, first=2)
    assert mask[:, 0].tolist() == [0, 0, 4, 12] and pos.tolist() == [-1, -1, 0, 1]


def test_masks_past_a_word():
    mask, pos = tree.masks([i - 1 for i in range(130)], 2, 5)
    assert [bin(int(x)).count("1") for x in mask[129]] == [64, 64] and pos[129] == 134
    assert int(mask[70, 1]) == (1 << 7) - 1


def test_a_chain_is_causal_attention():
    rng = np.random.default_rng(0)
    k, v, q = rng.normal(size=(9, 2, 8)), rng.normal(size=(9, 2, 8)), rng.normal(size=(4, 6, 8))
    mask, _ = tree.masks([-1, 0, 1, 2], 1, 5)
    out, mass, reach = tree.attend(q, k, v, tree.seen(mask, 9, 4), 0.3)
    ref = kv8.attend(q, k, v, [5, 6, 7, 8], 0.3)
    for a, b in zip((out, mass, reach), ref):
        assert np.array_equal(a, b)


def test_siblings_do_not_see_each_other():
    rng = np.random.default_rng(1)
    k, v, q = rng.normal(size=(5, 1, 4)), rng.normal(size=(5, 1, 4)), rng.normal(size=(3, 1, 4))
    mask, _ = tree.masks([-1, 0, 0], 1, 2)
    out = tree.attend(q, k, v, tree.seen(mask, 5, 3), 1.0)[0]
    at = [0, 1, 2, 4]
    assert np.allclose(out[2], kv8.attend(q[2:], k[at], v[at], [3], 1.0)[0][0])
    assert not tree.attend(q, k, v, np.zeros((3, 5), bool), 1.0)[0].any()


@pytest.mark.parametrize("context,keep", [(0, [1]), (5, [0, 2]), (14, [0, 1, 3, 9, 30]), (16, [2, 3, 20]), (31, [])])
def test_accept_keeps_values(context, keep):
    rng = np.random.default_rng(context)
    s = kv8.Kv8Sequence(2, 4)
    s.append(rng.normal(size=(context + 32, 2, 4)) * np.exp2(rng.integers(-3, 4, (context + 32, 1, 1))))
    before = s.values()
    n = tree.accept(s, context, keep)
    assert n == context + len(keep)
    want = before[list(range(context)) + [context + i for i in keep]]
    # a token keeps its four bits unless it lands among the subnormal codes of a larger scale
    step = np.repeat(s.scale, 16, 0)[:n, :, None] * 2.0 ** -10
    assert np.all(np.abs(s.values()[:n] - want) <= step)


def test_accept_of_a_prefix_moves_nothing():
    s = kv8.Kv8Sequence(1, 4)
    s.append(np.random.default_rng(0).normal(size=(40, 1, 4)))
    codes, scale = s.codes.copy(), s.scale.copy()
    assert tree.accept(s, 20, [0, 1, 2]) == 23
    assert np.array_equal(s.codes, codes) and np.array_equal(s.scale, scale)
