"""Plans, attention of drafted trees, appending and sampling rules together, as the example's rollout uses them."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as oracle
from paper_2510_11062_amd import rollout_example as ex
from tests.test_gpu_rollout_example import plain_norm_rope

TURN = 20


def setting(dev, dtype=torch.float32, E=3, seed=0):
    m = ex.make_model(dev, dtype, seed=seed)
    gen = torch.Generator().manual_seed(seed + 1)
    return m, [torch.randint(1, m.emb.shape[0], (18 + 21 * e,), generator=gen).to(dev) for e in range(E)]


def gumbel(m, n, seed=5):
    u = torch.rand(n, TURN, m.emb.shape[0], generator=torch.Generator().manual_seed(seed)).clamp(1e-6, 1 - 1e-6)
    return -torch.log(-torch.log(u)).to(m.emb.device)


def guesses_of(answer, share):
    """A draft whose better guesses are the true answer for a share of the candidates' places."""
    def draft(self, token):
        said = self.length.long()      # as many as there are tokens in the cache
        tree = [token]
        for j in range(1, self.T):
            at = (said + (j - 1) // 2).clamp(max=answer.shape[1] - 1)
            true = answer.gather(1, at[:, None])[:, 0]
            hit = (at * 7 + torch.arange(len(token), device=token.device)) % 10 < 10 * share
            tree.append(torch.where(hit & (j % 2 == 1), true, (true + j) % 2048))
        return torch.stack(tree, 1)
    return draft


@pytest.mark.gpu
@pytest.mark.parametrize("sampled", [False, True])
def test_drafts_change_the_steps_and_not_the_answers(gpu_device, monkeypatch, sampled):
    m, prompt = setting(gpu_device)
    noise = gumbel(m, 9) if sampled else None
    one = ex.roll_out_drafted(m, prompt, 3, TURN, 1, noise)
    assert one["steps"] == TURN
    for drafted, share in ((2, 1.0), (7, 1.0), (7, 0.7), (24, 0.8), (7, 0.0)):
        monkeypatch.setattr(ex.DraftedRollout, "draft", guesses_of(one["answer"], share))
        more = ex.roll_out_drafted(m, prompt, 3, TURN, drafted, noise)
        assert torch.equal(more["answer"], one["answer"]), drafted
        # of logits of order 10, in fp32, through kernels that add in other orders
        assert (more["logp"] - one["logp"]).abs().max() < 1e-3
        if share == 1.0:
            assert more["steps"] == -(-TURN // (1 + drafted // 2)), drafted
        elif share == 0:
            assert more["steps"] == TURN
        else:
            assert more["steps"] < TURN
    monkeypatch.undo()
    own = ex.roll_out_drafted(m, prompt, 3, TURN, 5, noise)
    assert torch.equal(own["answer"], one["answer"])


@pytest.mark.gpu
def test_every_choice_is_the_rules_best(gpu_device):
    """Against the model's plain pass over the whole answers and the rules in 64 bits."""
    m, prompt = setting(gpu_device)
    o = ex.roll_out_drafted(m, prompt, 3, TURN, 7)
    answer = o["answer"]
    said = torch.cat((torch.zeros(9, 1, dtype=torch.long, device=gpu_device), answer[:, :-1]), 1)
    with torch.no_grad():
        h = ex.hidden_states(m, [torch.cat((prompt[c // 3], said[c])) for c in range(9)], plain_norm_rope)
        logits = (h @ m.head.T).double().cpu().numpy()
    V, at = m.emb.shape[0], 0
    value = {k: float(o["settings"][k][0]) for k in ("repetition", "presence", "frequency", "temperature")}
    states = [np.arange(V) < V * 3 // 4, np.arange(V) >= V // 4]
    for c in range(9):
        at += len(prompt[c // 3])
        for t in range(TURN):
            out, lse, best, _ = oracle.sampling_row(logits[at], prompt[c // 3].tolist(), said[c, :t + 1].tolist(), *value.values(), {0: -5.0}, states[t % 2])
            got = int(answer[c, t])
            assert got == best or out[best] - out[got] < 1e-4, (c, t)      # of what fp32 leaves open
            assert abs(float(o["logp"][c, t]) - (out[got] - lse)) < 1e-3
            at += 1
    assert at == len(logits)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_pages_come_back(gpu_device, dtype):
    o = ex.run_drafted(dtype, E=2, K=3, turn=TURN, drafted=6)
    r = o["rollout"]
    assert torch.isfinite(o["logp"]).all() and (o["logp"] <= 0).all() and r.length.tolist() == [TURN] * 6
    held = [p for s in range(6) for p in r.pool.pages[s, :-(-TURN // ex.PAGE)].tolist()]
    held += [p for e, n in enumerate(r.prompt_len.tolist()) for p in r.prompts.pages[e, :-(-n // ex.PAGE)].tolist()]
    first, count = r.state.tolist()
    n = r.pool.ring.numel()
    free = [int(r.pool.ring[(first + i) % n]) for i in range(count)]
    assert sorted(held + free) == list(range(n))
    zero = torch.zeros_like(r.length)
    r._plan(r.pool, r.length, zero, 0, keep=zero)
    r._plan(r.prompts, r.prompt_len.clone(), torch.zeros_like(r.prompt_len), 0, keep=torch.zeros_like(r.prompt_len))
    assert int(r.state[1]) == n and int(r.data_error) == 0
