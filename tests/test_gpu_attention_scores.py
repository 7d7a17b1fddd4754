"""Attention where scores are far from 0: what one token has to itself by more than fp32's rounding of a score, and what equal tokens share."""
import numpy as np
import pytest
import torch

from oracle import rollout_oracle as oracle
from paper_2510_11062_amd import api
from tests.rollout_case import Paged, U16, U32, assert_within, host64, to_dev
from tests.test_gpu_tree_attention import bits, trees, wide

# Hq, Hk, D, page, lengths, new, group sizes, prefixes
SHAPES = {
    "one token each": (4, 2, 128, 16, [9, 30, 8, 64], [1, 1, 1, 1], [4], [197]),
    "few rows": (2, 2, 64, 16, [1, 17, 33, 65, 140], [1, 8, 5, 3, 2], [2, 3], [31, 300]),
    "wide groups": (8, 2, 128, 16, [33, 33, 70, 20, 64, 90], [30, 17, 64, 20, 1, 63], [5, 1], [700, 90]),
    "no groups": (4, 2, 64, 32, [64, 63, 300, 33], [64, 40, 33, 33], [], []),
    "head of 256": (4, 2, 256, 16, [50, 130, 17], [3, 40, 17], [3], [100]),
    "head of 80": (6, 2, 80, 16, [50, 33, 1], [20, 4, 1], [3], [100]),
    "long": (4, 1, 128, 64, [900, 64, 1500], [20, 64, 33], [3], [3000]),
}


LEVELS = (3e3, 3e8, 1e10, 1e33)      # of the queries' elements; a multiple of 2^32 is from some 1e9 on


def check(p, q, words, out, scale, what):
    """Scores are sums of D products in fp32: off by at most D 2^-24 sum_d |q_d k_d|.  Where the largest is ahead of all others by four times that and 60, the
    rest has no weight and out is that token's value (of tokens with the same key the mean of theirs, with bf16 each weight and the result are
    rounded); everywhere results are finite."""
    got, lse = host64(out["out"]), host64(out["lse"])
    clear = 0
    for s in range(len(p.length)):
        g, L, m, P = p.group[s], int(p.length[s]), int(p.new[s]), 0
        k, v = oracle.rows(p.k, p.pages[s], L), oracle.rows(p.v, p.pages[s], L)
        if g < len(p.size):
            P = int(p.prefix[g])
            k, v = np.concatenate([oracle.rows(p.k, p.prefix_pages[g], P), k]), np.concatenate([oracle.rows(p.v, p.prefix_pages[g], P), v])
        share, rows = q.shape[1] // k.shape[1], slice(p.cu_q[s], p.cu_q[s + 1])
        sees = np.ones((m, P + L), bool)
        for i in range(max(0, P + L - m), P + L):
            sees[:, i] = words[rows] >> np.uint64(i - (P + L - m)) & np.uint64(1) == 1
        for h in range(q.shape[1]):
            kk, vv, qq = k[:, h // share], v[:, h // share], q[rows, h]
            z, off = scale * (qq @ kk.T), scale * p.D * U32 * (np.abs(qq) @ np.abs(kk).T)
            z, off = np.where(sees, z, -np.inf), np.where(sees, off, 0).max(1)
            assert np.isfinite(got[rows, h]).all() and np.isfinite(lse[rows, h]).all(), what
            best = z.argmax(1)
            same = (kk[None] == kk[best][:, None]).all(2) & sees      # [m, tokens]
            ahead = z.max(1) - np.where(same, -np.inf, z).max(1, initial=-np.inf) >= 4 * off + 60
            clear += int(ahead.sum())
            n = same.sum(1)[:, None]
            want, size = same @ vv / n, same @ np.abs(vv) / n
            bound = (2.02 * U16 if p.dtype == torch.bfloat16 else 16 * U32) * size + 1e-30
            assert_within(got[rows, h][ahead], want[ahead], bound[ahead], what)
            assert (np.abs(lse[rows, h] - z.max(1)) <= off + np.log(n[:, 0]) + 8 * U32 * np.abs(z.max(1)) + 1e-6)[ahead].all(), what
    return clear, q.shape[0] * q.shape[1]


def cases(name, dtype, level, sign, seed):
    Hq, Hk, D, page, length, new, size, prefix = SHAPES[name]
    p = Paged(dtype, Hk, D, page, length, new, size, prefix, seed=seed)
    if sign:      # all scores of one sign
        p.k = np.abs(p.k)
    for s in range(len(length)):      # a sequence's first two tokens have one key: where it is ahead they share
        if length[s] - new[s] > 1:
            at = [(int(p.pages[s][i // page]), i % page) for i in (0, 1)]
            p.k[at[1][0], :, at[1][1]] = p.k[at[0][0], :, at[0][1]]
    q = p.queries(Hq)
    q = to_dev((sign * np.abs(q) if sign else q) * level, p.dtype, "cpu").double().numpy()
    return p, q


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", SHAPES)
@pytest.mark.parametrize("sign", [0, 1, -1])
def test_trees(gpu_device, dtype, name, sign):
    seen = 0
    for level in LEVELS:
        p, q = cases(name, dtype, level, sign, 3)
        words = trees(p.rs, p.new, "paths")
        for kv in (p.device(gpu_device), wide(p.device(gpu_device))):
            out = api.at_grpo_tree_attention(kv, to_dev(q, p.dtype, gpu_device), bits(words, gpu_device), max_q=int(p.new.max()), want_lse=True)
            clear, rows = check(p, q, words, out, p.D ** -0.5, f"{level}")
            assert 4 * clear > rows
            seen += clear
    assert seen


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", SHAPES)
@pytest.mark.parametrize("sign", [0, 1, -1])
def test_an_order(gpu_device, dtype, name, sign):
    for level in LEVELS:
        p, q = cases(name, dtype, level, sign, 4)
        words = trees(p.rs, p.new, "order")
        for max_q in {1, int(p.new.max()), 4096}:
            out = api.at_grpo_prefix_attention(p.device(gpu_device), to_dev(q, p.dtype, gpu_device), max_q=max_q, want_lse=True)
            clear, rows = check(p, q, words, out, p.D ** -0.5, f"{level} max_q={max_q}")
            assert 4 * clear > rows


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_every_size_beside_each_other(gpu_device, dtype):
    """A row's scores are its own: beside rows of any size the small ones are what they are alone, bit for bit."""
    Hq, Hk, D, page, length, new, size, prefix = SHAPES["wide groups"]
    p = Paged(dtype, Hk, D, page, length, new, size, prefix, seed=6)
    q = to_dev(p.queries(Hq), p.dtype, gpu_device)
    words = bits(trees(p.rs, p.new, "paths"), gpu_device)
    large = torch.arange(len(q), device=gpu_device) % 3 == 1
    mixed = torch.where(large[:, None, None], q.float() * 1e14, q.float()).to(q.dtype)
    for kv in (p.device(gpu_device), wide(p.device(gpu_device))):
        call = lambda x: api.at_grpo_tree_attention(kv, x, words, want_lse=True)
        want, got = call(q), call(mixed)
        assert torch.equal(got["out"][~large], want["out"][~large]) and torch.equal(got["lse"][~large], want["lse"][~large])
        assert bool(torch.isfinite(got["out"]).all())
