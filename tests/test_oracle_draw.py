"""The sampling oracle against cases worked out by hand."""
import math

import numpy as np
import pytest

from oracle.draw import Row, weight_slack

Z = np.log([0.1, 0.4, 0.2, 0.2, 0.1])     # order: 1, 2, 3, 0, 4


def test_everything_is_drawn_by_id():
    r = Row(Z)
    assert [r.draw(u)[0] for u in (0.0, 0.09, 0.11, 0.49, 0.51, 0.69, 0.71, 0.89, 0.91, 0.999)] == [0, 0, 1, 1, 2, 2, 3, 3, 4, 4]
    assert np.allclose([r.draw(0.3)[1], r.draw(0.3)[2]], math.log(0.4))


@pytest.mark.parametrize("settings,ids", [
    (dict(top_k=1), [1]), (dict(top_k=2), [1, 2]), (dict(top_k=3), [1, 2, 3]), (dict(top_k=9), [0, 1, 2, 3, 4]),
    (dict(top_p=0.39), [1]), (dict(top_p=0.41), [1, 2]), (dict(top_p=0.61), [1, 2, 3]), (dict(top_p=0.81), [0, 1, 2, 3]),
    (dict(top_p=1e-9), [1]), (dict(min_p=0.3), [1, 2, 3]), (dict(min_p=0.2), [0, 1, 2, 3, 4]), (dict(min_p=1.0), [1]),
    # top-p's share is of what top-k left: 0.4 of 0.8 and 0.6 of 0.8
    (dict(top_k=3, top_p=0.49), [1]), (dict(top_k=3, top_p=0.51), [1, 2]), (dict(top_k=3, top_p=0.76), [1, 2, 3]),
    (dict(top_k=4, top_p=0.99, min_p=0.6), [1]), (dict(temperature=0.0, top_k=3), [1])])
def test_what_is_kept(settings, ids):
    z = Z + (1e-9 if "min_p" in settings and settings["min_p"] < 1 else 0) * np.array([1, 0, 1, 1, 1])
    r = Row(z, **settings)
    assert r.kept(r.low).tolist() == ids
    share = np.exp(z[ids]) / np.exp(z[ids]).sum()
    for i, (a, b) in enumerate(zip(np.cumsum(share) - share, np.cumsum(share))):
        t, lp, kp = r.draw((a + b) / 2)
        assert t == ids[i] and math.isclose(kp, math.log(share[i]), abs_tol=1e-9)
        assert np.allclose(r.span(t, r.low), (a, b))


def test_temperature():
    r = Row(Z, temperature=2.0)
    p = np.sqrt(np.exp(Z)) / np.sqrt(np.exp(Z)).sum()
    assert np.allclose([r.draw(u)[1] for u in (0.01, 0.3)], np.log(p[:2]))


def test_masked_logits_are_never_drawn():
    r = Row([-np.inf, 0.0, -np.inf, 0.0])
    assert [r.draw(u)[0] for u in (0.0, 0.49, 0.51, 0.99)] == [1, 1, 3, 3]


def test_slack():
    assert 2e-12 < weight_slack([0.0], 1.0) < 3e-12
    r = Row(Z, top_p=0.6, slack=1e-6)
    assert (r.low, r.high) == (2, 3)
