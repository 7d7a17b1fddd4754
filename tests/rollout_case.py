"""Batches of sequences in a paged cache, on the host and on the GPU, and the oracle's results for them."""
from __future__ import annotations

import numpy as np
import torch

from oracle import rollout_oracle as oracle
from paper_2510_11062_amd import api

U16 = 2.0 ** -8      # largest relative error of rounding to bf16 (8 significant bits, to nearest)
U32 = 2.0 ** -24

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def rounded(a, dtype):
    """The values as the dtype holds them, in 64 bits."""
    return torch.from_numpy(np.asarray(a, dtype=np.float64)).to(dtype).double().numpy()


def to_dev(a, dtype, dev):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).to(dev)


def i32(a, dev):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(dev)


def host64(t):
    return t.detach().double().cpu().numpy()


class Paged:
    """Sequences with `length` own tokens (`new` of them new), in groups of `size` behind prefixes of `prefix` tokens."""

    def __init__(self, dtype, Hk, D, page, length, new=None, size=(), prefix=(), seed=0, spare_columns=1, fill=float("nan")):
        self.dtype, self.Hk, self.D, self.page = DTYPES[dtype], Hk, D, page
        self.length = np.array(length, dtype=np.int64)
        self.decode = new is None
        self.new = np.ones(len(length), dtype=np.int64) if new is None else np.array(new, dtype=np.int64)
        self.size, self.prefix = np.array(size, dtype=np.int64), np.array(prefix, dtype=np.int64)
        n_seq, n_group = len(self.length), len(self.size)
        assert n_group == 0 or self.size.sum() <= n_seq
        rs = self.rs = np.random.default_rng(seed)
        cols = lambda x: (int(max(x)) + page - 1) // page if len(x) else 0
        used = [-(-int(x) // page) for x in list(self.length) + list(self.prefix)]
        self.n_pages = sum(used) + 2
        order = rs.permutation(self.n_pages)
        # entries behind a sequence's last page are not read: page ids that no cache has stand there
        self.pages = np.full((n_seq, cols(self.length) + spare_columns), 1 << 30, dtype=np.int64)
        self.prefix_pages = np.full((n_group, cols(self.prefix) + spare_columns), -(1 << 30), dtype=np.int64)
        at = 0
        for i, u in enumerate(used):
            (self.pages[i] if i < n_seq else self.prefix_pages[i - n_seq])[:u] = order[at:at + u]
            at += u
        self.group_seq = np.concatenate([[0], np.cumsum(self.size)])
        self.cu_q = np.concatenate([[0], np.cumsum(self.new)])
        self.group = np.searchsorted(self.group_seq[1:], np.arange(n_seq), side="right")
        self.before = np.array([self.prefix[g] if g < n_group else 0 for g in self.group], dtype=np.int64)
        shape = (self.n_pages, Hk, page, D)
        self.k, self.v = (rounded(rs.normal(size=shape), self.dtype) for _ in range(2))
        # what no sequence's tokens occupy holds NaN
        used_place = np.zeros((self.n_pages, page), dtype=bool)
        for table, n in [(self.pages[s], self.length[s]) for s in range(n_seq)] + [(self.prefix_pages[g], self.prefix[g]) for g in range(n_group)]:
            for i in range(int(n)):
                used_place[table[i // page], i % page] = True
        for c in (self.k, self.v):
            c.transpose(0, 2, 1, 3)[~used_place] = fill

    @property
    def n_tok(self):
        return int(self.new.sum())

    def device(self, dev, **over):
        t = dict(cache_k=to_dev(self.k, self.dtype, dev), cache_v=to_dev(self.v, self.dtype, dev), pages=i32(self.pages, dev),
                 length=i32(self.length, dev), cu_q=None if self.decode else i32(self.cu_q, dev))
        if len(self.size):
            t.update(group_seq=i32(self.group_seq, dev), prefix_len=i32(self.prefix, dev), prefix_pages=i32(self.prefix_pages, dev))
        t.update(over)
        return api.KVBatch(**t)

    def queries(self, Hq, scale=1.0):
        return rounded(self.rs.normal(size=(self.n_tok, Hq, self.D)) * scale, self.dtype)

    def attention(self, q, scale, causal=True):
        """The oracle's (out, lse, mag, big, n): n [tokens] visible tokens of each query."""
        out, mag = np.zeros(q.shape), np.zeros(q.shape)
        lse, big = np.full(q.shape[:2], -np.inf), np.zeros(q.shape[:2])
        n = np.zeros(len(q), dtype=np.int64)
        for s in range(len(self.length)):
            a, b = self.cu_q[s], self.cu_q[s + 1]
            g, L, m = self.group[s], int(self.length[s]), int(self.new[s])
            k, v = oracle.rows(self.k, self.pages[s], L), oracle.rows(self.v, self.pages[s], L)
            if g < len(self.size):
                P = int(self.prefix[g])
                k = np.concatenate([oracle.rows(self.k, self.prefix_pages[g], P), k])
                v = np.concatenate([oracle.rows(self.v, self.prefix_pages[g], P), v])
            seen = [int(self.before[s]) + (max(0, L - m + j + 1) if causal else L) for j in range(m)]
            out[a:b], lse[a:b], mag[a:b], big[a:b] = oracle.attention(q[a:b], k, v, scale, seen)
            n[a:b] = seen
        return out, lse, mag, big, n


def attention_bounds(dtype, D, out, mag, big, n):
    """Largest errors of out and lse.  A score is a sum of D products, whose rounding errors add up like a random walk of
    sqrt(D) steps of 2^-24 of its terms' size; the sums over n tokens likewise; four standard deviations.  bf16 rounds the weights (each by
    at most 2^-8 of itself) and the result."""
    z = 4 * U32 * (4 + 2 * np.sqrt(D)) * big
    walk = 4 * U32 * (8 + 2 * np.sqrt(np.maximum(n, 1)))[:, None]
    rel = 2 * z + walk
    o = rel[..., None] * mag
    if dtype == torch.bfloat16:
        o = o + U16 * (mag + np.abs(out)) * (1 + rel[..., None])
    return o + 1e-30, rel


def assert_within(got, ref, bound, what):
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == ref.shape, what
    bad = ~(np.abs(got - ref) <= bound)
    if bad.any():
        at = tuple(int(x) for x in np.argwhere(bad)[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} outside, first at {at}: {got[at]} for {ref[at]}, bound {np.broadcast_to(bound, ref.shape)[at]}")
