"""Scratch memory of the calls in front of the head: it holds no error word, and the words of the calls that have one outlive it."""
import pytest
import torch

from paper_2510_11062_amd import api
from tests.rollout_case import Paged, to_dev


def attention(dev):
    p = Paged("bf16", 2, 64, 16, [40, 7], None, [2], [30], seed=1)
    kv, q = p.device(dev), to_dev(p.queries(4), p.dtype, dev)
    return lambda: api.at_grpo_prefix_attention(kv, q)


def gradient(dev):
    x, w = torch.randn(30, 4, 64, device=dev), torch.ones(64, device=dev)
    return lambda: api.at_grpo_qk_norm_rope_bwd(x, None, x, None, None, None, w)


@pytest.mark.gpu
@pytest.mark.parametrize("make", [attention, gradient])
def test_no_error_word_is_read_from_it(gpu_device, make):
    out = make(gpu_device)()
    with pytest.raises(api.AtGrpoError, match="data_error"):
        api.error_word(out["workspace"])


@pytest.mark.gpu
@pytest.mark.parametrize("make", [attention, gradient])
def test_the_words_of_other_calls_stay(gpu_device, make):
    call = make(gpu_device)
    ids = torch.zeros(4, dtype=torch.int32, device=gpu_device)
    reward = torch.tensor([1.0, float("nan"), 0.0, 2.0], device=gpu_device)
    out = api.at_grpo_group_advantage(ids, ids, ids, reward, 1, 1, 1)
    assert api.error_word(out["workspace"]) == 2      # AT_GRPO_DATA_REWARD
    call()
    assert api.error_word(out["workspace"]) == 2
    api.at_grpo_group_advantage(ids, ids, ids, reward.nan_to_num(), 1, 1, 1)
    call()
    assert api.error_word(out["workspace"]) == 0


@pytest.mark.gpu
def test_scratch_follows_the_workspace(gpu_device):
    """Grown by another call, or released: the next call has scratch of the one in use, and the same results."""
    call = attention(gpu_device)
    want = call()["out"].clone()
    api.release_workspace()
    first = call()
    assert torch.equal(first["out"], want)
    grown = first["workspace"].numel() * 2
    api._workspace(grown, gpu_device)
    second = call()
    assert torch.equal(second["out"], want) and second["workspace"].numel() > first["workspace"].numel()
    api.release_workspace()
