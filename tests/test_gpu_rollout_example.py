"""The example's rollout and training step, which run all the calls in front of the head together."""
import pytest
import torch

from paper_2510_11062_amd import rollout_example as ex


def plain_norm_rope(q, k, q_norm, k_norm, rope, position):
    turn = rope[position.long()].to(q.dtype)[:, None]

    def one(x, w):
        u = x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + 1e-6) * w
        a, b = u.chunk(2, -1)
        return torch.cat((a * turn[..., 0] - b * turn[..., 1], b * turn[..., 0] + a * turn[..., 1]), -1)

    return one(q, q_norm), one(k, k_norm)


@pytest.mark.gpu
def test_rollout_and_training_agree(gpu_device):
    # fp32 throughout: what the two passes round differently is some 2^-24 of sums of up to 512 terms, and two layers pass it on
    r = ex.run(torch.float32)
    assert r["apart"] < 1e-4
    mask = r["roll"]["mask"].bool()
    logp = r["step"]["logp"].view(mask.shape)
    assert (logp - r["roll"]["logp"])[mask].abs().max() < 1e-3      # of logits of order 10
    got = [{k: w[k].grad.clone() for k in w} for w in r["model"].layers]
    m = ex.make_model(gpu_device, torch.float32)
    ex.train_step(m, r["prompt"], 4, r["roll"], r["reward"], norm_rope=plain_norm_rope)
    for w, g in zip(m.layers, got):
        for name in w:
            assert (w[name].grad - g[name]).norm() < 1e-3 * w[name].grad.norm(), name
            assert g[name].norm() > 0


@pytest.mark.gpu
def test_bf16(gpu_device):
    # roundings of 2^-9 on average at a dozen places of a layer, two layers, add up like a random walk
    r = ex.run(torch.bfloat16, E=2, K=3)
    assert r["apart"] < 3e-2
    assert torch.isfinite(r["step"]["d_hidden"].float()).all() and all(torch.isfinite(w["wq"].grad.float()).all() for w in r["model"].layers)
