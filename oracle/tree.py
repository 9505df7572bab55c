"""Float64 reference of drafted trees over a key/value cache: what a node sees,
its position, attention under a mask, and the move of an accepted path.

Node i of a tree lies in slot context + i of its sequence; nodes before `first`
are padding (a sequence with fewer tokens than rows)."""
from __future__ import annotations

import numpy as np

from . import kv8


def paths(parent, first: int = 0):
    """For each node, itself and its ancestors in ascending order; None for padding, for a node whose parent is none
    and for what is behind such a one."""
    out = []
    for i, p in enumerate(parent):
        if i < first or not -1 <= p < i:
            out.append(None)
        elif p < first:                                # the context, or a padding row
            out.append([i])
        else:
            out.append(None if out[p] is None else out[p] + [i])
    return out


def masks(parent, words: int, context: int, first: int = 0):
    """(mask uint64 [n, words], position [n])."""
    mask, pos = np.zeros((len(parent), words), np.uint64), np.full(len(parent), -1)
    for i, p in enumerate(paths(parent, first)):
        if p is None:
            continue
        for j in p:
            if j < 64 * words:
                mask[i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
        pos[i] = context + len(p) - 1
    return mask, pos


def seen(mask, tokens: int, nodes: int):
    """[nodes, tokens] truth values: the tokens of a sequence (its nodes are the last ones) that each node sees."""
    mask = np.asarray(mask, np.uint64)
    c0 = tokens - nodes
    out = np.zeros((nodes, tokens), bool)
    for i in range(nodes):
        if c0 + i < 0:
            continue
        out[i, :max(c0, 0)] = True
        for j in range(min(nodes, 64 * mask.shape[1])):
            if c0 + j >= 0:
                out[i, c0 + j] = bool(mask[i, j // 64] >> np.uint64(j % 64) & np.uint64(1))
    return out


def attend(q, k, v, sees, scale):
    """q [rows, n_q, dims]; k, v [tokens, n_kv, dims]; sees [rows, tokens].  Returns the outputs (zeros where nothing is
    seen), sum_j p_j |v_j| and the largest sum_d |q_d k_jd| of what is seen."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    rep = q.shape[1] // k.shape[1]
    out, mass, reach = np.zeros_like(q), np.zeros_like(q), np.zeros(q.shape[:2])
    for r in range(len(q)):
        at = np.flatnonzero(sees[r])
        if not len(at):
            continue
        for h in range(q.shape[1]):
            kk, vv = k[at, h // rep], v[at, h // rep]
            s = kk @ q[r, h] * scale
            w = np.exp(s - s.max())
            w /= w.sum()
            out[r, h], mass[r, h] = w @ vv, w @ np.abs(vv)
            reach[r, h] = (np.abs(kk) @ np.abs(q[r, h])).max()
    return out, mass, reach


def accept(seq: kv8.Kv8Sequence, context: int, keep, first: int = 0):
    """Moves the nodes `keep` (ascending numbers) of a Kv8Sequence behind the context; returns the tokens that are left.
    Codes behind them stay as they are, as do blocks that receive no token."""
    src = list(range(context)) + [context - first + i for i in keep]
    codes, scale = seq.codes.copy(), seq.scale.copy()
    values = kv8.e4m3_values()
    for b in range(-(-len(src) // kv8.BLOCK)):
        t = range(b * kv8.BLOCK, min((b + 1) * kv8.BLOCK, len(src)))
        if all(src[i] == i for i in t):
            continue
        for h in range(codes.shape[1]):
            old = [seq.scale[src[i] // kv8.BLOCK, h] for i in t]
            scale[b, h] = max(old)
            for i, s in zip(t, old):
                codes[i, h] = kv8.e4m3_round(values[seq.codes[src[i], h]] * (s / scale[b, h]))
    seq.codes, seq.scale = codes, scale
    return len(src)
