"""Candidates of shared prompts, rolled out and trained on with the library's calls, in a small model of attention layers and a head.

    python -m paper_2510_11062_amd.rollout_example [--dtype f32] [--envs E] [--candidates K] [--drafted T]

Rollout: every prompt goes into the paged caches once, K candidates answer it token by token behind that prefix, all are given a message
of several tokens (an environment's observation, as between two turns), and answer again.  Training: the same tokens in one pass with
gradients, grouped advantages, the policy loss and its backward through the head and the layers, the update of the head.

    at_grpo_kv_append          prompts, single tokens, messages: keys and values into the cache, queries rotated
    at_grpo_prefix_attention   the same three
    at_grpo_qk_norm_rope, _bwd the training pass, as one autograd function
    at_grpo_group_advantage, at_grpo_policy_loss_fwd_bwd, at_grpo_head_update

With --drafted an answer is first rolled out T drafted tokens at a time: every candidate gets a tree of guesses, all are attended at once, the
sampling rules choose a token behind each, and the path that the guesses share with the choices is kept.

    at_grpo_kv_plan            pages, places and positions of prompts and trees, and the pages of what was not kept back
    at_grpo_tree_attention     the trees
    at_grpo_logit_rules        penalties, biases, a grammar's masks and temperature on the logits behind every drafted token

Plain products (projections, logits to sample from) and the training pass's attention are torch's; random weights, synthetic prompts.
"""
from __future__ import annotations

import argparse
import time
from dataclasses import dataclass, field
from typing import List

import torch

from . import api

PAGE = 16


@dataclass
class Model:
    emb: torch.Tensor                 # [V, H]
    head: torch.Tensor                # [V, H]
    layers: List[dict] = field(default_factory=list)      # wq [Hq D, H], wk and wv [Hk D, H], wo [H, Hq D], q_norm and k_norm [D]
    rope: torch.Tensor = None
    Hq: int = 0
    Hk: int = 0
    D: int = 0


def make_model(dev, dtype, V=2048, H=256, Hq=8, Hk=2, D=64, layers=2, positions=1024, seed=0) -> Model:
    gen = torch.Generator().manual_seed(seed)
    rand = lambda *shape, std=1.0: (std * torch.randn(*shape, generator=gen)).to(dtype).to(dev)
    m = Model(rand(V, H), rand(V, H, std=H ** -0.5), Hq=Hq, Hk=Hk, D=D, rope=api.at_grpo_rope_table(positions, D, base=1e4, device=dev))
    for _ in range(layers):
        m.layers.append(dict(wq=rand(Hq * D, H, std=H ** -0.5), wk=rand(Hk * D, H, std=H ** -0.5), wv=rand(Hk * D, H, std=H ** -0.5),
                             wo=rand(H, Hq * D, std=(Hq * D) ** -0.5), q_norm=1 + rand(D, std=0.1), k_norm=1 + rand(D, std=0.1)))
    return m


def _qkv(m: Model, w: dict, x):
    return (x @ w["wq"].T).view(-1, m.Hq, m.D), (x @ w["wk"].T).view(-1, m.Hk, m.D), (x @ w["wv"].T).view(-1, m.Hk, m.D)


# ---- rollout ----------------------------------------------------------------------------------------
class Rollout:
    """The caches of all layers, the prompts' pages and the candidates'."""

    def __init__(self, m: Model, prompt_len, K: int, most: int):
        self.m, self.K = m, K
        dev, E = m.emb.device, len(prompt_len)
        self.prompt_len = torch.tensor(prompt_len, dtype=torch.int32, device=dev)
        cols_p, cols = -(-max(prompt_len) // PAGE), -(-most // PAGE)
        n_pages = E * cols_p + E * K * cols
        ids = torch.randperm(n_pages, generator=torch.Generator().manual_seed(1)).to(torch.int32).to(dev)
        self.prefix_pages, self.pages = ids[:E * cols_p].view(E, cols_p), ids[E * cols_p:].view(E * K, cols)
        self.group_seq = torch.arange(0, E * K + 1, K, dtype=torch.int32, device=dev)
        self.length = torch.zeros(E * K, dtype=torch.int32, device=dev)
        self.caches = [tuple(torch.empty(n_pages, m.Hk, PAGE, m.D, dtype=m.emb.dtype, device=dev) for _ in range(2)) for _ in m.layers]
        self.data_error = torch.zeros(1, dtype=torch.int32, device=dev)

    def _layers(self, token, kv_of, max_q):
        """Hidden states of new tokens: appended and attended layer by layer."""
        m, x = self.m, self.m.emb[token]
        for w, cache in zip(m.layers, self.caches):
            kv = kv_of(*cache)
            q, k, v = _qkv(m, w, x)
            api.at_grpo_kv_append(kv, q, k, v, m.rope, w["q_norm"], w["k_norm"], q_out=q, data_error=self.data_error)
            a = api.at_grpo_prefix_attention(kv, q, max_q=max_q, data_error=self.data_error)["out"]
            x = x + a.view(-1, m.Hq * m.D) @ w["wo"].T
        return x

    def prompts(self, token, cu):
        """The prompts, whole; their pages become the prefixes."""
        return self._layers(token, lambda k, v: api.KVBatch(k, v, self.prefix_pages, self.prompt_len, cu_q=cu), int(self.prompt_len.max()))

    def step(self, token):
        """One token of every candidate, or with token [candidates, n] n of them."""
        n = 1 if token.dim() == 1 else token.shape[1]
        cu = None if n == 1 else torch.arange(0, token.numel() + 1, n, dtype=torch.int32, device=token.device)
        self.length += n
        return self._layers(token.reshape(-1), lambda k, v: api.KVBatch(k, v, self.pages, self.length, cu_q=cu, group_seq=self.group_seq,
                                                                        prefix_len=self.prompt_len, prefix_pages=self.prefix_pages), n)


@torch.no_grad()
def roll_out(m: Model, prompt, K: int, turn: int, message):
    """prompt: the prompts' tokens, a tensor for each.  Two turns of `turn` tokens with `message` [tokens] between them.  Returns what went in
    (`token` [candidates, n]), what was drawn (`drawn`, meaningful where `mask`), its log-probabilities, and the hidden states."""
    dev, E = m.emb.device, len(prompt)
    gen = torch.Generator(device=dev).manual_seed(2)
    r = Rollout(m, [len(p) for p in prompt], K, 2 * turn + len(message))
    cu = torch.tensor([0] + [len(p) for p in prompt], device=dev).cumsum(0).to(torch.int32)
    r.prompts(torch.cat(prompt), cu)
    token, drawn, logp, mask, hidden = [], [], [], [], []

    def draw(h):
        lp = torch.log_softmax(h.float() @ m.head.float().T, -1)
        y = torch.multinomial(lp.exp(), 1, generator=gen)
        return y[:, 0], lp.gather(1, y)[:, 0]

    x = torch.zeros(E * K, dtype=torch.long, device=dev)      # token 0 begins an answer
    for part in range(2):
        for _ in range(turn):
            h = r.step(x)
            y, lp = draw(h)
            token.append(x[:, None]), drawn.append(y[:, None]), logp.append(lp[:, None]), hidden.append(h[:, None])
            mask.append(torch.ones_like(y, dtype=torch.uint8)[:, None])
            x = y
        if part == 0:
            given = message.expand(E * K, -1)
            h = r.step(given).view(E * K, len(message), -1)
            token.append(given), drawn.append(given), hidden.append(h)
            logp.append(torch.zeros(given.shape, device=dev)), mask.append(torch.zeros(given.shape, dtype=torch.uint8, device=dev))
    error = int(r.data_error)
    if error:
        raise api.AtGrpoError(f"data errors {error:#x} in the rollout")
    cat = lambda xs: torch.cat(xs, 1)
    return dict(token=cat(token), drawn=cat(drawn), logp=cat(logp), mask=cat(mask), hidden=cat(hidden))


# ---- drafted tokens -----------------------------------------------------------------------------------
class DraftedRollout:
    """Candidates of shared prompts that answer `drafted` tokens at a time."""

    def __init__(self, m: Model, prompt, K: int, most: int, drafted: int):
        dev, E = m.emb.device, len(prompt)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
        self.m, self.K, self.T, self.n = m, K, drafted, E * K
        # a tree: a token's two best guesses hang on it, and on the better of them its two best, and so on
        self.parent = [-1] + [max(0, (j - 1) // 2 * 2 - 1) for j in range(1, drafted)]
        cols_p, cols = -(-max(map(len, prompt)) // PAGE), -(-(most + drafted) // PAGE)
        n_pages = E * cols_p + E * K * cols
        self.group_seq, self.prompt_len = torch.arange(0, E * K + 1, K, dtype=torch.int32, device=dev), i32([len(p) for p in prompt])
        ring = torch.randperm(n_pages, generator=torch.Generator().manual_seed(1)).to(torch.int32).to(dev)
        table = lambda rows, width: torch.zeros(rows, width, dtype=torch.int32, device=dev)
        self.state = i32([0, n_pages])
        self.prompts = api.PagePool(table(E, cols_p), ring, PAGE)
        self.pool = api.PagePool(table(E * K, cols), ring, PAGE, group_seq=self.group_seq, prefix_len=self.prompt_len)
        self.caches = [tuple(torch.zeros(n_pages, m.Hk, PAGE, m.D, dtype=m.emb.dtype, device=dev) for _ in range(2)) for _ in m.layers]
        self.data_error = i32([0])
        self.length = torch.zeros(E * K, dtype=torch.int32, device=dev)      # tokens of the candidates in the cache
        self.prompt = torch.zeros(E, max(map(len, prompt)), dtype=torch.int32, device=dev)
        for row, p in zip(self.prompt, prompt):
            row[:len(p)] = p

    def _plan(self, pool, length, add, n_tok, **kw):
        return api.at_grpo_kv_plan(pool, length, add, self.state, n_tok, length_out=length, state_out=self.state, data_error=self.data_error, **kw)

    def read_prompts(self):
        """The prompts go into the cache; what the candidates begin with comes behind them."""
        m, tokens = self.m, torch.cat([row[:n] for row, n in zip(self.prompt, self.prompt_len.tolist())]).long()
        length = torch.zeros_like(self.prompt_len)
        plan = self._plan(self.prompts, length, self.prompt_len, len(tokens))
        x = m.emb[tokens]
        for w, cache in zip(m.layers, self.caches):
            kv = api.KVBatch(*cache, self.prompts.pages, length, cu_q=plan["cu_q"])
            q, k, v = _qkv(m, w, x)
            api.at_grpo_kv_append(kv, q, k, v, m.rope, w["q_norm"], w["k_norm"], q_out=q, data_error=self.data_error)
            a = api.at_grpo_prefix_attention(kv, q, max_q=int(self.prompt_len.max()), data_error=self.data_error)["out"]
            x = x + a.view(-1, m.Hq * m.D) @ w["wo"].T

    def draft(self, token):
        """Trees [candidates, T] behind the tokens [candidates] that were chosen last: by what the head makes of a token's embedding alone."""
        tree = [token]
        for j in range(1, self.T):
            guesses = torch.topk(self.m.emb[tree[self.parent[j]]].float() @ self.m.head.float().T, 2).indices
            tree.append(guesses[:, (j - 1) % 2])
        return torch.stack(tree, 1)

    def attend(self, tree):
        """Hidden states behind every token of the trees, the plan, and the keys and values that went into the cache."""
        m, n_tok = self.m, tree.numel()
        add = torch.full_like(self.length, self.T)
        parent = torch.tensor(self.parent * self.n, dtype=torch.int32, device=tree.device)
        plan = self._plan(self.pool, self.length, add, n_tok, parent=parent)
        rows, x = [], m.emb[tree.reshape(-1)]
        for w, cache in zip(m.layers, self.caches):
            kv = api.KVBatch(*cache, self.pool.pages, self.length, cu_q=plan["cu_q"], group_seq=self.group_seq, prefix_len=self.prompt_len,
                             prefix_pages=self.prompts.pages)
            q, k, v = _qkv(m, w, x)
            turned = api.at_grpo_qk_norm_rope(q, k, m.rope, plan["position"], w["q_norm"], w["k_norm"], data_error=self.data_error)      # by depth, not by place
            api.at_grpo_kv_append(kv, None, turned["k"], v, None, data_error=self.data_error)
            a = api.at_grpo_tree_attention(kv, turned["q"], plan["ancestors"], max_q=self.T, data_error=self.data_error)["out"]
            x = x + a.view(-1, m.Hq * m.D) @ w["wo"].T
            rows.append((turned["k"], v))
        return x, plan, rows

    def keep(self, path, rows):
        """Of the trees' tokens those of `path` [candidates, T] (a mask) stay, one behind the other; the others' pages go back."""
        count = path.sum(1).to(torch.int32)
        at = path.reshape(-1).nonzero()[:, 0]
        start = torch.cat((count.new_zeros(1), count.cumsum(0).to(torch.int32)))
        kept = self.length - self.T + count
        for cache, (k, v) in zip(self.caches, rows):
            kv = api.KVBatch(*cache, self.pool.pages, kept, cu_q=start, group_seq=self.group_seq, prefix_len=self.prompt_len, prefix_pages=self.prompts.pages)
            api.at_grpo_kv_append(kv, None, k[at], v[at], None, data_error=self.data_error)
        self._plan(self.pool, self.length, torch.zeros_like(self.length), 0, keep=kept)


def sampling_rules(m: Model, n: int):
    """Settings of n candidates: penalties, a temperature, a bias against token 0, and a grammar of two states (odd places take the first three
    quarters of the vocabulary, even ones the last three)."""
    dev, V = m.emb.device, m.emb.shape[0]
    full = lambda x: torch.full((n,), x, device=dev)
    allowed = torch.zeros(2, -(-V // 32) * 32, dtype=torch.int64, device=dev)
    allowed[0, :V * 3 // 4] = allowed[1, V // 4:V] = 1
    words = (allowed.view(2, -1, 32) << torch.arange(32, device=dev)).sum(2)
    return dict(repetition=full(1.2), presence=full(0.2), frequency=full(0.1), temperature=full(0.8),
                bias_cu=torch.arange(n + 1, dtype=torch.int32, device=dev), bias_token=torch.zeros(n, dtype=torch.int32, device=dev), bias=full(-5.0),
                allowed=torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32))


@torch.no_grad()
def roll_out_drafted(m: Model, prompt, K: int, turn: int, drafted: int, noise=None):
    """Answers of `turn` tokens by every candidate, `drafted` at a time.  noise [candidates, turn, V]: added to the logits of each place, of which
    the largest is chosen (Gumbel noise draws from the distribution); None: the best token.  Returns tokens [candidates, turn], their
    log-probabilities, steps, and the rollout."""
    r = DraftedRollout(m, prompt, K, turn + 1, drafted)
    r.read_prompts()
    dev, n, T = m.emb.device, r.n, drafted
    settings = sampling_rules(m, n)
    cand = torch.arange(n, device=dev)
    answer = torch.zeros(n, turn, dtype=torch.long, device=dev)
    logp = torch.zeros(n, turn, device=dev)
    said = torch.zeros(n, dtype=torch.long, device=dev)                 # tokens chosen so far
    token = torch.zeros(n, dtype=torch.long, device=dev)                # token 0 begins an answer
    history = torch.zeros(n, turn, dtype=torch.int32, device=dev)     # what a candidate has in the cache
    parent = torch.tensor(r.parent, device=dev)
    steps = 0
    while int(said.min()) < turn:
        tree = r.draft(token)
        before = r.length.clone()
        h, plan, rows = r.attend(tree)
        place = (said[:, None] + plan["position"].view(n, T) - plan["position"].view(n, T)[:, :1]).clamp(max=turn - 1)     # of the token that comes behind each
        rules = api.LogitRules(tokens=history, length=before, prompt=r.prompt, prompt_len=r.prompt_len, group_seq=r.group_seq, cu_q=plan["cu_q"],
                               drafted=tree.reshape(-1).to(torch.int32), ancestors=plan["ancestors"], mask_row=(place % 2).reshape(-1).to(torch.int32), **settings)
        o = api.at_grpo_logit_rules(rules, h @ m.head.T, out_dtype=torch.float32, data_error=r.data_error)
        choice = o["best"].long() if noise is None else (o["out"] + noise[cand[:, None], place].view(n * T, -1)).argmax(1)
        lp = (o["out"].gather(1, choice[:, None])[:, 0] - o["lse"]).view(n, T)
        choice = choice.view(n, T)
        # from the root on, as long as a guess is what was chosen
        path, at = torch.zeros(n, T, dtype=torch.bool, device=dev), torch.zeros(n, dtype=torch.long, device=dev)
        alive = said < turn
        for _ in range(T):
            path[cand[alive], at[alive]] = True
            history[cand[alive], (before + path.sum(1) - 1)[alive]] = tree[cand, at][alive].to(torch.int32)
            answer[cand[alive], said[alive]], logp[cand[alive], said[alive]] = choice[cand, at][alive], lp[cand, at][alive]
            token = torch.where(alive, choice[cand, at], token)
            said = said + alive
            child = (parent == at[:, None]) & (tree == token[:, None])
            alive = alive & child.any(1) & (said < turn)
            at = torch.where(alive, child.float().argmax(1), at)
        r.keep(path, rows)
        steps += 1
    error = int(r.data_error)
    if error:
        raise api.AtGrpoError(f"data errors {error:#x} in the rollout")
    return dict(answer=answer, logp=logp, steps=steps, rollout=r, settings=settings)


# ---- training ---------------------------------------------------------------------------------------
class NormRope(torch.autograd.Function):
    """at_grpo_qk_norm_rope and its gradient."""

    @staticmethod
    def forward(ctx, q, k, q_norm, k_norm, rope, position):
        ctx.save_for_backward(q, k, q_norm, k_norm, rope, position)
        out = api.at_grpo_qk_norm_rope(q, k, rope, position, q_norm, k_norm)
        return out["q"], out["k"]

    @staticmethod
    def backward(ctx, dq, dk):
        q, k, q_norm, k_norm, rope, position = ctx.saved_tensors
        g = api.at_grpo_qk_norm_rope_bwd(dq.contiguous(), dk.contiguous(), q, k, rope, position, q_norm, k_norm)
        return g["dq"], g["dk"], g["dq_weight"].to(q_norm.dtype), g["dk_weight"].to(k_norm.dtype), None, None


def _attention(q, k, v, share):
    """Causal attention of one sequence, in float32: q [n, Hq, D], k and v [n, Hk, D]."""
    q, k, v = (x.float().transpose(0, 1).contiguous() for x in (q, k.repeat_interleave(share, 1), v.repeat_interleave(share, 1)))
    s = torch.matmul(q, k.transpose(1, 2).contiguous()) * q.shape[-1] ** -0.5
    s = s.masked_fill(torch.ones(s.shape[1:], dtype=torch.bool, device=s.device).triu(1), float("-inf"))
    return torch.matmul(torch.softmax(s, -1), v).transpose(0, 1)


def hidden_states(m: Model, sequences, norm_rope=NormRope.apply):
    """Hidden states of whole sequences, with gradients."""
    sizes = [len(s) for s in sequences]
    position = torch.cat([torch.arange(n, dtype=torch.int32, device=m.emb.device) for n in sizes])
    x = m.emb[torch.cat(sequences)]
    for w in m.layers:
        q, k, v = _qkv(m, w, x)
        q, k = norm_rope(q, k, w["q_norm"], w["k_norm"], m.rope, position)
        a = torch.cat([_attention(*t, m.Hq // m.Hk) for t in zip(q.split(sizes), k.split(sizes), v.split(sizes))])
        x = x + a.to(x.dtype).reshape(len(x), -1) @ w["wo"].T
    return x


def train_step(m: Model, prompt, K: int, roll: dict, reward, lr=1e-3, norm_rope=NormRope.apply):
    """One step on a rollout: gradients stay at the layers' weights (`grad`), the head is updated in place."""
    dev, (R, n) = m.emb.device, roll["token"].shape
    for w in m.layers:
        for name in w:
            w[name] = w[name].detach().requires_grad_()
    x = hidden_states(m, [torch.cat([prompt[s // K], roll["token"][s]]) for s in range(R)], norm_rope)
    ends = torch.tensor([len(prompt[s // K]) + n for s in range(R)]).cumsum(0).tolist()
    h = torch.cat([x[e - n:e] for e in ends])

    env = torch.arange(R, dtype=torch.int32, device=dev) // K
    zero = torch.zeros_like(env)
    adv = api.at_grpo_group_advantage(env, zero, zero, reward, len(prompt), 1, 1)["adv"]
    batch = api.Batch(h.detach(), [m.head], roll["drawn"].reshape(-1).to(torch.int32), torch.arange(0, R * n + 1, n, device=dev),
                      mask=roll["mask"].reshape(-1).contiguous())
    step = api.at_grpo_policy_loss_fwd_bwd(batch, roll["logp"].reshape(-1).contiguous(), adv, 0.2, 0.2)
    h.backward(step["d_hidden"])
    moments = [torch.zeros_like(step["dW"][0]) for _ in range(2)]
    master = None if m.head.dtype == torch.float32 else [m.head.float()]
    api.at_grpo_head_update([m.head], step["dW"], [moments[0]], [moments[1]], 1, W_master=master, lr=lr)
    return dict(step, hidden=h.detach().view(R, n, -1), adv=adv)


def run(dtype=torch.bfloat16, E=3, K=4, turn=12, device="cuda", seed=0, say=lambda s: None):
    m = make_model(device, dtype, seed=seed)
    gen = torch.Generator().manual_seed(seed + 1)
    V = m.emb.shape[0]
    draw = lambda n: torch.randint(1, V, (n,), generator=gen).to(device)
    prompt = [draw(20 + 17 * e) for e in range(E)]
    message = draw(21)
    t0 = time.time()
    roll = roll_out(m, prompt, K, turn, message)
    say(f"rollout: {E} prompts, {E * K} candidates, {roll['token'].shape[1]} tokens each, {time.time() - t0:.2f} s")
    reward = ((roll["drawn"] % 2 == 0) * roll["mask"]).sum(1).float() / (2 * turn)      # answers of even tokens
    step = train_step(m, prompt, K, roll, reward)
    torch.cuda.synchronize()
    apart = float((step["hidden"].double() - roll["hidden"].double()).norm() / roll["hidden"].double().norm())
    norms = [float(w[name].grad.float().norm()) for w in m.layers for name in ("wq", "q_norm", "k_norm")]
    say(f"training: loss {float(step['loss'][0]):+.5f}, hidden states {apart:.1e} from the rollout's, "
        f"gradient norms {', '.join(f'{x:.1e}' for x in norms)}")
    return dict(model=m, prompt=prompt, roll=roll, reward=reward, step=step, apart=apart)


def run_drafted(dtype=torch.bfloat16, E=3, K=4, turn=24, drafted=7, device="cuda", seed=0, say=lambda s: None):
    m = make_model(device, dtype, seed=seed)
    gen = torch.Generator().manual_seed(seed + 1)
    prompt = [torch.randint(1, m.emb.shape[0], (20 + 17 * e,), generator=gen).to(device) for e in range(E)]
    noise = -torch.log(-torch.log(torch.rand(E * K, turn, m.emb.shape[0], generator=gen).clamp(1e-9, 1 - 1e-7))).to(device)
    t0 = time.time()
    o = roll_out_drafted(m, prompt, K, turn, drafted, noise)
    torch.cuda.synchronize()
    say(f"drafted rollout: {E * K} candidates, {turn} tokens each in {o['steps']} steps of {drafted}, {time.time() - t0:.2f} s, "
        f"log-probability {float(o['logp'].mean()):+.3f} a token")
    return dict(o, model=m, prompt=prompt, noise=noise)


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    p.add_argument("--envs", type=int, default=3)
    p.add_argument("--candidates", type=int, default=4)
    p.add_argument("--drafted", type=int, default=0)
    a = p.parse_args()
    if a.drafted:
        run_drafted({"bf16": torch.bfloat16, "f32": torch.float32}[a.dtype], a.envs, a.candidates, drafted=a.drafted, say=lambda s: print(s, flush=True))
    run({"bf16": torch.bfloat16, "f32": torch.float32}[a.dtype], a.envs, a.candidates, say=lambda s: print(s, flush=True))
