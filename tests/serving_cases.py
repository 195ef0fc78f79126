"""Small paged batches for the serving operators' tests: made on the host,
checked against oracle.serving."""
from __future__ import annotations

import numpy as np
import torch

import oracle.serving as sv
import paper_2609_00224_amd as q

TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def rounded(x, name):
    """x as the type's values, fp64."""
    return torch.from_numpy(np.ascontiguousarray(x)).to(TORCH[name]).double().numpy()


class Paged:
    """Sequences of (length, new tokens) in a shuffled pool.  `k`, `v`: the
    cached values [length][heads][dim] of each sequence, fp64 and exact."""

    def __init__(self, rng, lens, heads, dim, page, fmt, extra_pages=3, spread=1.0):
        self.lens, self.heads, self.dim, self.page, self.fmt = lens, heads, dim, page, fmt
        need = [-(-max(c, 0) // page) for c, _ in lens]
        self.pages = sum(need) + extra_pages
        order = rng.permutation(self.pages).astype(np.int32)
        self.table = np.full((len(lens), max(1, max(need))), -1, np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at:at + n]
            at += n
        self.kv_len = np.array([c for c, _ in lens], np.int32)
        self.q_start = np.concatenate([[0], np.cumsum([n for _, n in lens])]).astype(np.int32)
        self.rows = int(self.q_start[-1])
        self.pool, self.values = {}, {}
        for w in ("k", "v"):
            x = rng.standard_normal((self.pages, heads, page, dim)) * spread
            if fmt in ("f16", "bf16"):
                vals = rounded(x, fmt)
                self.pool[w] = (torch.from_numpy(vals).to(TORCH[fmt]), None)
            else:
                x = rounded(x, "f16")
                code, scale = sv.encode(x, fmt)
                vals = sv.decode(code, scale, fmt)
                self.pool[w] = (torch.from_numpy(pack(code, fmt)), torch.from_numpy(scale))
            self.values[w] = vals
        self.k, self.v = ([self.sequence(w, s) for s in range(len(lens))] for w in ("k", "v"))

    def places(self, s, first, last):
        t = np.arange(first, last)
        return self.table[s, t // self.page], t % self.page

    def sequence(self, w, s):
        pg, off = self.places(s, 0, max(0, int(self.kv_len[s])))
        return self.values[w][pg, :, off]

    def cache(self):
        dev = {w: tuple(None if t is None else t.cuda() for t in self.pool[w]) for w in ("k", "v")}
        return q.KvCache(self.fmt, dev["k"][0], dev["v"][0], dev["k"][1], dev["v"][1])

    def meta(self):
        return tuple(torch.from_numpy(x).cuda() for x in (self.q_start, self.kv_len, self.table))


def pack(code, fmt):
    return code if fmt == "e4m3" else (code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8)


# Relative half steps of the 16-bit types.
HALF = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def attention_reference(p, Q, scale, window=0):
    """(out, bound) of a batch, Q [rows][q heads][dim] fp64.

    The bound on |kernel - out|, per element: the result's own rounding, u
    |out|; the weights' rounding to the 16-bit type, u times the weights' mean
    of |v| (the sum of the weights is not rounded); the fp32 scores: each a sum
    of dim products, off by at most (dim + 2) 2^-24 sum|q k| scale before and 4
    ulps of exp2 after, which moves a weight by that share and the quotient by
    twice it; fp16 weights below 2^-14 of the running unit are off by 2^-25 each
    where the largest is at least 2^6; fp16's smallest step, 2^-25."""
    u = HALF[p.qtype]
    group = Q.shape[1] // p.heads
    out, bound = np.zeros_like(Q), np.zeros_like(Q)
    for s, (c, n) in enumerate(p.lens):
        rows = slice(p.q_start[s], p.q_start[s + 1])
        pos = np.arange(c - n, c)
        for a in range(Q.shape[1]):
            k, v = p.k[s][:, a // group], p.v[s][:, a // group]
            o, spread = sv.attention(Q[rows, a], k, v, pos, scale, window)
            out[rows, a] = o
            if not len(k):
                continue
            score = (np.abs(Q[rows, a]) @ np.abs(k).T).max(-1, keepdims=True) * scale
            share = 2 * (score * (p.dim + 2) * 2.0 ** -24 + 4 * 2.0 ** -23 + c * 2.0 ** -24)
            bound[rows, a] = u * np.abs(o) + (u + share) * spread * 1.01 + c * 2.0 ** -31 * np.abs(v).max() + 2.0 ** -25
    return out, bound
