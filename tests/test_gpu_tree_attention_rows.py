"""Trees of drafted tokens behind rows of nobody, and over keys that are infinite: every row that is served, against the oracle."""
import numpy as np
import pytest
import torch

from paper_2510_11062_amd import api
from tests.rollout_case import Paged, to_dev
from tests.test_gpu_tree_attention import attention, bits, check, trees, wide


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [[4, 8, 2, 0], [40, 64, 9, 12]])
@pytest.mark.parametrize("tables", ["near", "wide"])
@pytest.mark.parametrize("front,behind", [(1, 0), (2, 0), (0, 3), (2, 5)])
def test_rows_of_nobody_in_front_and_behind(gpu_device, dtype, new, tables, front, behind):
    """cu_q begins behind the first rows and ends in front of the last: those get 0 and -inf, the others are the sequences', and nothing is wrong."""
    p = Paged(dtype, 2, 128, 16, [60, 100, 33, 64], new, [2], [50], seed=7)
    p.cu_q = p.cu_q + front
    n = int(p.cu_q[-1]) + behind
    words = np.full(n, (1 << 64) - 1, np.uint64)
    words[front:n - behind] = trees(p.rs, p.new, "paths")
    q64 = to_dev(p.rs.normal(size=(n, 4, 128)), p.dtype, "cpu").double().numpy()
    kv, word = p.device(gpu_device), torch.zeros(1, dtype=torch.int32, device=gpu_device)
    kv = wide(kv) if tables == "wide" else kv
    for max_q in {1, max(new), 4096}:
        out = api.at_grpo_tree_attention(kv, to_dev(q64, p.dtype, gpu_device), bits(words, gpu_device), max_q=max_q, want_lse=True, data_error=word)
        check(p, out, attention(p, q64, words, 128 ** -0.5), f"max_q={max_q}")
        nobody = list(range(front)) + list(range(n - behind, n))
        assert bool((out["out"][nobody] == 0).all()) and bool(torch.isneginf(out["lse"][nobody]).all()) and int(word) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [[4, 8, 2, 0], [40, 64, 9, 12]])
@pytest.mark.parametrize("tables", ["near", "wide"])
def test_a_sequence_that_begins_in_the_first_rows(gpu_device, dtype, new, tables):
    """Its rows in front of cu_q[0] are nobody's, and the next is its first new token, with fewer of them."""
    p = Paged(dtype, 2, 128, 16, [60, 100, 33, 64], new, [2], [50], seed=7)
    n = p.n_tok
    p.cu_q[0], p.new[0] = 2, p.new[0] - 2
    words = np.zeros(n, np.uint64)
    words[2:] = trees(p.rs, p.new, "order")
    q64 = to_dev(p.rs.normal(size=(n, 4, 128)), p.dtype, "cpu").double().numpy()
    kv, word = p.device(gpu_device), torch.zeros(1, dtype=torch.int32, device=gpu_device)
    kv = wide(kv) if tables == "wide" else kv
    out = api.at_grpo_tree_attention(kv, to_dev(q64, p.dtype, gpu_device), bits(words, gpu_device), max_q=max(new), want_lse=True, data_error=word)
    check(p, out, attention(p, q64, words, 128 ** -0.5))
    assert bool((out["out"][:2] == 0).all()) and bool(torch.isneginf(out["lse"][:2]).all()) and int(word) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,new", [(2, [5, 8, 6]), (8, [9, 40, 64])])
@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("tables", ["near", "wide"])
@pytest.mark.parametrize("value", [-np.inf, np.inf])
def test_infinite_keys_of_tokens_that_are_seen(gpu_device, dtype, Hq, new, grouped, tables, value):
    """A key whose element 3 is infinite: its score is infinite with the sign of the query's element.  At -inf the token has no weight, as if the
    row's bit were not set, and the row is what it is without it, bit for bit; at inf it is inf - inf, NaN.  Rows that do not see it stay."""
    p = Paged(dtype, 2, 64, 16, [20, 70, 64], new, *(([2], [45]) if grouped else ()), seed=2)
    words = trees(p.rs, new, "paths")
    q64 = p.queries(Hq)
    assert (q64[..., 3] != 0).all()
    q = to_dev(q64, p.dtype, gpu_device)
    kv = p.device(gpu_device)
    kv = wide(kv) if tables == "wide" else kv
    call = lambda w: api.at_grpo_tree_attention(kv, q, bits(w, gpu_device), max_q=max(new), want_lse=True)
    want = call(words & ~np.uint64(4))      # nobody sees the third drafted token
    whole, met = call(words), []
    for s in range(3):
        at = int(p.length[s] - p.new[s]) + 2
        page, place = int(p.pages[s][at // 16]), at % 16
        mine = np.zeros(len(words), bool)
        mine[p.cu_q[s]:p.cu_q[s + 1]] = True
        sees = torch.from_numpy(mine & (words >> np.uint64(2) & np.uint64(1) == 1)).to(gpu_device)
        old = kv.cache_k[page, :, place].clone()
        kv.cache_k[page, :, place, 3] = float(value)
        got = call(words)
        kv.cache_k[page, :, place] = old
        for name in ("out", "lse"):
            assert torch.equal(got[name][~sees], whole[name][~sees]), (s, name)
        low = sees[:, None] & ((q[..., 3] > 0) == (value < 0))      # rows and heads
        high = sees[:, None] & ~low
        assert torch.equal(got["out"][low], want["out"][low]) and torch.equal(got["lse"][low], want["lse"][low]), s
        assert bool(torch.isnan(got["out"][high]).all()) and bool(torch.isnan(got["lse"][high]).all()), s
        met += [int(low.sum()), int(high.sum())]
    assert sum(met[::2]) and sum(met[1::2])      # both signs, over all sequences
