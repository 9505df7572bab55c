"""Float64 reference of sampling with temperature, top-k, top-p and min-p from a
given uniform number."""
from __future__ import annotations

import math

import numpy as np


class Row:
    """One row of logits and its settings: the order of its tokens (by logit, then id), their weights, and how many of
    the first are kept.  ``slack``: a relative error of sums of weights that decisions may have; ``low`` and ``high`` are
    then the fewest and the most tokens that top-p may keep."""

    def __init__(self, z, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, slack=0.0):
        z = np.asarray(z, np.float64)
        self.z, self.top = z, z.max()
        self.t = 1.0 if temperature == 0 else float(temperature)
        x = (z - self.top) / self.t
        self.w = np.exp(x)
        self.total = self.w.sum()
        self.order = np.argsort(-z, kind="stable")
        n = len(z) if top_k <= 0 else min(top_k, len(z))
        self.low = self.high = n
        if top_p < 1:
            w = self.w[self.order[:n]]
            before, all_ = np.cumsum(w) - w, w.sum()
            self.low = max(1, int((before < (top_p - slack) * all_).sum()))
            self.high = max(1, int((before < (top_p + slack) * all_).sum()))
        if min_p > 0:
            m = int((z >= self.top + self.t * math.log(min(min_p, 1.0))).sum())
            self.low, self.high = min(self.low, m), min(self.high, m)
        if temperature == 0:
            self.low = self.high = 1

    def kept(self, n):
        """Ids of the first n, ascending."""
        return np.sort(self.order[:n])

    def draw(self, u, n=None):
        """(token, log-probability, log-probability among the kept n)."""
        ids = self.kept(self.low if n is None else n)
        run = np.cumsum(self.w[ids])
        i = int(np.searchsorted(run, u * run[-1], side="right"))
        return self.logs(int(ids[min(i, len(ids) - 1)]), self.low if n is None else n)

    def logs(self, token, n):
        x = (self.z[token] - self.top) / self.t
        return token, x - math.log(self.total), x - math.log(self.w[self.order[:n]].sum())

    def span(self, token, n):
        """The shares of u for which a token of the kept n is drawn: (from, to)."""
        ids = self.kept(n)
        run = np.cumsum(self.w[ids])
        i = int(np.searchsorted(ids, token))
        return (run[i] - self.w[token]) / run[-1], run[i] / run[-1]


def weight_slack(z, temperature):
    """Relative error of a sum of weights that are each within 2e-12 of their value, or whole numbers of 2^-42 of the
    largest weight (each off by half of one)."""
    return 2e-12 + len(z) * 2.0 ** -43
