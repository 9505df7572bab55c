"""Helpers of the 8-bit cache's tests: batches of sequences with oracle caches
beside a device cache, and the layout of a block written out."""
from __future__ import annotations

import numpy as np
import torch

from oracle import kv8

BF16, F32 = torch.bfloat16, torch.float32
UNIT = {BF16: 2.0 ** -8, F32: 2.0 ** -24}     # half a step, relative


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def host(t):
    return t.detach().double().cpu().numpy()


def rounded(a, dtype):
    """Values of `dtype` as float64."""
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).double().numpy()


class Batch:
    """Sequences with oracle keys and values, a scattered page table and a device cache; `spare` pages belong to
    nobody.  The device cache starts full of `fill` (a code) under scale 1."""

    def __init__(self, old, n_kv, hd, page=16, capacity=None, seed=0, spare=3, fill=0x7F):
        import paper_2606_02218_amd as rg
        self.rng = np.random.default_rng(seed)
        self.n_kv, self.hd, self.page, S = n_kv, hd, page, len(old)
        self.width = -(-(capacity or max(max(old), 1) + 64) // page)
        self.pages = S * self.width + spare
        self.tab = self.rng.permutation(self.pages)[:S * self.width].reshape(S, self.width).astype(np.int32)
        self.k = [kv8.Kv8Sequence(n_kv, hd) for _ in old]
        self.v = [kv8.Kv8Sequence(n_kv, hd) for _ in old]
        self.cache = rg.Kv8Cache.empty(self.pages, n_kv, hd, page)
        for t in self.cache[:2]:
            t.view(torch.uint8).fill_(fill)
        for t in self.cache[2:]:
            t.fill_(1.0)
        for s, n in enumerate(old):
            if n:
                self.k[s].append(rounded(self.rng.normal(0, 1.0, (n, n_kv, hd)), F32))
                self.v[s].append(rounded(self.rng.normal(0, 1.0, (n, n_kv, hd)), F32))
        self.write()

    def blocks(self, seq, keys):
        """The oracle's codes as device blocks [blocks, n_kv, 16 * hd] (slots behind the end left as None mask)."""
        n = len(seq.codes)
        nb = -(-n // 16)
        c = np.zeros((nb * 16, self.n_kv, self.hd), np.uint8)
        c[:n] = seq.codes
        mask = np.zeros((nb * 16, self.n_kv, self.hd), bool)
        mask[:n] = True

        def lay(a):
            a = a.reshape(nb, 16, self.n_kv, self.hd).transpose(0, 2, 1, 3)                  # [nb, kv, t, d]
            if keys:
                a = a.reshape(nb, self.n_kv, 16, self.hd // 16, 16).transpose(0, 1, 3, 2, 4)
            else:
                a = a.reshape(nb, self.n_kv, 4, 4, self.hd).transpose(0, 1, 2, 4, 3)
            return a.reshape(nb, self.n_kv, 16 * self.hd)
        return lay(c), lay(mask)

    def places(self, s, nb):
        b = np.arange(nb)
        return self.tab[s][b * 16 // self.page], b % (self.page // 16)

    def write(self):
        """The oracle's caches into the device cache."""
        for seqs, t, sc in ((self.k, self.cache.k, self.cache.k_scale), (self.v, self.cache.v, self.cache.v_scale)):
            codes, scale = t.view(torch.uint8).cpu().numpy(), sc.cpu().numpy()
            for s, seq in enumerate(seqs):
                c, m = self.blocks(seq, seqs is self.k)
                pg, sub = self.places(s, len(c))
                codes[pg, :, sub] = np.where(m, c, codes[pg, :, sub])
                scale[pg, :, sub] = seq.scale[:len(c)]
            t.view(torch.uint8).copy_(torch.from_numpy(codes))
            sc.copy_(torch.from_numpy(scale))

    def image(self, only=None):
        """(codes, scales) of keys and of values that the device cache should hold, given what it holds elsewhere now."""
        out = []
        for seqs, t, sc in ((self.k, self.cache.k, self.cache.k_scale), (self.v, self.cache.v, self.cache.v_scale)):
            codes, scale = t.view(torch.uint8).cpu().numpy().copy(), sc.cpu().numpy().copy()
            for s, seq in enumerate(seqs):
                if only is not None and s not in only:
                    continue
                c, m = self.blocks(seq, seqs is self.k)
                pg, sub = self.places(s, len(c))
                codes[pg, :, sub] = np.where(m, c, codes[pg, :, sub])
                scale[pg, :, sub] = seq.scale[:len(c)]
            out += [codes, scale]
        return out

    def snapshot(self):
        return [self.cache.k.view(torch.uint8).cpu().numpy().copy(), self.cache.k_scale.cpu().numpy().copy(),
                self.cache.v.view(torch.uint8).cpu().numpy().copy(), self.cache.v_scale.cpu().numpy().copy()]

    def logical(self, s, n, keys):
        """Values that the device cache holds for the first n tokens of sequence s."""
        t, sc = (self.cache.k, self.cache.k_scale) if keys else (self.cache.v, self.cache.v_scale)
        nb = -(-n // 16)
        pg, sub = self.places(s, nb)
        c = kv8.e4m3_values()[t.view(torch.uint8).cpu().numpy()[pg, :, sub]] * sc.cpu().numpy().astype(np.float64)[pg, :, sub][..., None]
        if keys:
            c = c.reshape(nb, self.n_kv, self.hd // 16, 16, 16).transpose(0, 3, 1, 2, 4)
        else:
            c = c.reshape(nb, self.n_kv, 4, self.hd, 4).transpose(0, 2, 4, 1, 3)
        return c.reshape(nb * 16, self.n_kv, self.hd)[:n]

    def lengths(self):
        return np.array([len(s.codes) for s in self.k], np.int32)


def offsets(new):
    return dev(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))


def attention_bound(ref, mass, reach, hd, n, scale, dtype, p_step):
    """Largest error of an attention output, elementwise.  Scores are sums of hd products in fp32: at most
    (hd + 8) 2^-24 sum|q k| scale off, and turning them into exp2's argument rounds at 2^-23 of their size; twice that
    moves a probability relatively (numerator and sum), with 2^-22 of the exponential itself.  Sums of n terms round at
    n 2^-24 of sum p|v| (and of the sum p).  p_step: half a step of the probabilities' own rounding."""
    e = ((hd + 8) * 2.0 ** -24 + 2.0 ** -22) * reach[..., None] * scale + 2.0 ** -21 + n * 2.0 ** -23
    return UNIT[dtype] * np.abs(ref) * 1.01 + mass * (2 * e + p_step)
