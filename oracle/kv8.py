"""Float64 reference of the rotary positions and of the 8-bit paged key/value
cache: what a sequence's cache holds after appends, and attention over it.

Codes are e4m3: sign, 4 exponent bits (bias 7), 3 fraction bits; exponent 0 is
subnormal (fraction * 2^-9), the code with all seven lower bits set is NaN,
448 the largest value, no infinities.  A block of 16 tokens of one head has a
scale 2^e; a value is code * 2^e.
"""
from __future__ import annotations

import numpy as np

BLOCK = 16
MAX = 448.0


def e4m3_values() -> np.ndarray:
    """The value of each of the 256 codes."""
    b = np.arange(256)
    exp, frac = (b >> 3) & 15, (b & 7).astype(np.float64)
    v = np.where(exp == 0, frac * 2.0 ** -9, (1.0 + frac / 8.0) * 2.0 ** (exp - 7.0))
    v = np.where((b & 127) == 127, np.nan, v)
    return np.where(b >= 128, -v, v)


_VALUES = e4m3_values()
_POS = _VALUES[:127]


def e4m3_round(x) -> np.ndarray:
    """Codes nearest to x, ties to the even code; larger magnitudes saturate, NaN is code 255."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(np.nan_to_num(x, nan=0.0, posinf=MAX, neginf=MAX)), MAX)
    hi = np.searchsorted(_POS, a)                  # first value >= a
    lo = np.maximum(hi - 1, 0)
    up, down = _POS[hi] - a, a - _POS[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.signbit(x), code + 128, code)
    return np.where(np.isnan(x), 255, code).astype(np.uint8)


def block_exponent(x) -> int:
    """The least e in [-64, 119] with 448 * 2^e >= the largest finite magnitude."""
    a = np.abs(np.asarray(x, np.float64))
    m = float(np.max(np.where(np.isfinite(a), a, 0.0), initial=0.0))
    e = -64
    while e < 119 and MAX * 2.0 ** e < m:
        e += 1
    return e


class Kv8Sequence:
    """One sequence's keys or values: codes [tokens, heads, dims] and, per block and head, scales."""

    def __init__(self, heads: int, dims: int):
        self.codes = np.zeros((0, heads, dims), np.uint8)
        self.scale = np.zeros((0, heads))

    def append(self, x):
        """x: [rows, heads, dims] in float64, as one call's rows."""
        x = np.asarray(x, np.float64)
        start, n = len(self.codes), len(x)
        self.codes = np.concatenate([self.codes, np.zeros(x.shape, np.uint8)])
        blocks = -(-(start + n) // BLOCK)
        self.scale = np.concatenate([self.scale, np.zeros((blocks - len(self.scale), x.shape[1]))])
        for b in range(start // BLOCK, blocks if n else start // BLOCK):
            lo, hi = max(start, b * BLOCK), min(start + n, (b + 1) * BLOCK)
            for h in range(x.shape[1]):
                new = x[lo - start:hi - start, h]
                s = 2.0 ** block_exponent(new)
                if lo > b * BLOCK:
                    old = self.scale[b, h]
                    s = max(s, old)
                    stay = self.codes[b * BLOCK:lo, h]
                    if s > old:
                        self.codes[b * BLOCK:lo, h] = e4m3_round(_VALUES[stay] * (old / s))
                self.codes[lo:hi, h] = e4m3_round(new / s)
                self.scale[b, h] = s

    def values(self) -> np.ndarray:
        return _VALUES[self.codes] * np.repeat(self.scale, BLOCK, 0)[:len(self.codes), :, None]


def frequencies(rot: int, theta: float, scaling=None, factor=1.0, length=0.0, slow=1.0, fast=32.0):
    """Angles per position of the rot/2 pairs, and the amplitude of cos and sin."""
    i = np.arange(rot // 2, dtype=np.float64)
    if scaling == "base":
        theta = theta * factor ** (rot / (rot - 2.0))
    w = theta ** (-2.0 * i / rot)
    if scaling == "linear":
        w = w / factor
    if scaling == "bands":
        turns = w * length / (2.0 * np.pi)
        g = np.clip((turns - slow) / (fast - slow), 0.0, 1.0)
        return w * (g + (1.0 - g) / factor), 0.1 * np.log(factor) + 1.0
    return w, 1.0


def rotate(x, cos, sin, layout: str = "half", inverse: bool = False) -> np.ndarray:
    """x [rows, heads, dims] with each row's cos and sin [rows, pairs]."""
    x = np.asarray(x, np.float64)
    c, s = np.asarray(cos, np.float64)[:, None], np.asarray(sin, np.float64)[:, None] * (-1.0 if inverse else 1.0)
    m = c.shape[-1]
    a, b = (slice(0, m), slice(m, 2 * m)) if layout == "half" else (slice(0, 2 * m, 2), slice(1, 2 * m, 2))
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def attend(q, k, v, pos, scale):
    """q [rows, n_q, dims] at positions pos; k, v [tokens, n_kv, dims].  Returns the outputs and, for error
    bounds, sum_j p_j |v_j| and the largest sum_d |q_d k_jd| of every row and head."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    rep = q.shape[1] // k.shape[1]
    out, mass, reach = np.zeros_like(q), np.zeros_like(q), np.zeros(q.shape[:2])
    for r, p in enumerate(pos):
        if p < 0:
            continue
        for h in range(q.shape[1]):
            kk, vv = k[:p + 1, h // rep], v[:p + 1, h // rep]
            s = kk @ q[r, h] * scale
            w = np.exp(s - s.max())
            w /= w.sum()
            out[r, h], mass[r, h] = w @ vv, w @ np.abs(vv)
            reach[r, h] = (np.abs(kk) @ np.abs(q[r, h])).max()
    return out, mass, reach


class Kv8Model:
    """The oracle decoder with its keys and values in 8 bits.  ``jitter``: relative noise on keys and values before they
    are stored, to see what a computation in fewer bits may do to the codes."""

    def __new__(cls, shape, weights, jitter: float = 0.0, seed: int = 0):
        from .model import OracleModel

        class Model(OracleModel):
            def new_cache(self):
                s = self.s
                return [{"k": Kv8Sequence(s.n_kv_heads, s.head_dim), "v": Kv8Sequence(s.n_kv_heads, s.head_dim)}
                        for _ in range(s.n_layers)]

            @staticmethod
            def copy_cache(cache):
                out = []
                for c in cache:
                    d = {}
                    for n, q in c.items():
                        d[n] = Kv8Sequence(0, 0)
                        d[n].codes, d[n].scale = q.codes.copy(), q.scale.copy()
                    out.append(d)
                return out

            def noisy(self, a):
                return a * (1.0 + jitter * rng.standard_normal(a.shape)) if jitter else a

            def forward(self, tokens, positions, cache):
                s = self.s
                tokens, positions = np.asarray(tokens, np.int64), np.asarray(positions, np.int64)
                T = len(tokens)
                x = np.asarray(self.embed[tokens], np.float64)
                for lw, c in zip(self.layers, cache):
                    h = self.rmsnorm(x, lw["attn_norm"])
                    q = self.rope(self.linear(h, lw["wq"]).reshape(T, s.n_q_heads, s.head_dim), positions)
                    k = self.rope(self.linear(h, lw["wk"]).reshape(T, s.n_kv_heads, s.head_dim), positions)
                    v = self.linear(h, lw["wv"]).reshape(T, s.n_kv_heads, s.head_dim)
                    c["k"].append(self.noisy(k))
                    c["v"].append(self.noisy(v))
                    o = self.attention(q, c["k"].values(), c["v"].values(), positions, np.arange(len(c["k"].codes)))
                    x = x + self.linear(o.reshape(T, s.q_dim), lw["wo"])
                    h2 = self.rmsnorm(x, lw["ffn_norm"])
                    x = x + self.linear(self.silu(self.linear(h2, lw["w_gate"])) * self.linear(h2, lw["w_up"]), lw["w_down"])
                return self.linear(self.rmsnorm(x, self.final_norm), self.lm_head)

            def decode_batch(self, tokens, positions, caches):
                return np.concatenate([self.forward([t], [p], c) for t, p, c in zip(tokens, positions, caches)])

        rng = np.random.default_rng(seed)
        return Model(shape, weights)
