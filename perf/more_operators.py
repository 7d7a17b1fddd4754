"""The operators around a rollout that drafts its tokens, as cases that can be timed and compared: pages and slots from the sequences'
lengths, attention of trees of drafted tokens over the paged cache, and the rules of sampling on the logits that come out.

A case is a dict of plain values; `prepare` builds on the GPU what a rollout holds before the call, `run` is one pass, through the library's
entry points where `own` is true and in elementary torch operations where it is not.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False


def listed():
    return [
        # one token for each of the 4 candidates of one turn: latency
        dict(name="plan-turn", kind="plan", groups=1, K=4, prefix=197, held=32, add=1, page=16, keep="all", tree=False),
        # up to 1536 candidates (C3's number of responses) with up to 16 drafted tokens each; of the last step's most were not accepted, and
        # some candidates have ended
        dict(name="plan-drafts", kind="plan", groups=192, K=8, prefix=600, held=900, add=16, page=16, keep="some", tree=True),
        # the first turn's prompts of C4's 256 environments and 2 agents, of up to 1100 tokens
        dict(name="plan-prompts", kind="plan", groups=0, K=512, prefix=0, held=0, add=1100, page=64, keep="all", tree=False),
        # 8 drafted tokens for each of the 4 candidates of one turn, a short prompt: latency
        dict(name="tree-turn", kind="tree", dtype="bf16", groups=1, K=4, prefix=197, own=32, queries=8, hq=16, hk=8, D=128, page=16),
        # 32 prompts of up to 2400 tokens, up to 8 candidates of each with responses of lognormal lengths, up to 16 drafted tokens
        dict(name="tree-rollout", kind="tree", dtype="bf16", groups=32, K=8, prefix=2400, own=1500, queries=16, hq=32, hk=8, D=128, page=16),
        # two long prompts (a history of many turns), 8 candidates of each, up to 32 drafted tokens
        dict(name="tree-long", kind="tree", dtype="bf16", groups=2, K=8, prefix=40000, own=512, queries=32, hq=16, hk=8, D=128, page=64),
        # 24 conversations of up to 9000 tokens that share nothing, large trees, many queries on few keys
        dict(name="tree-alone", kind="tree", dtype="bf16", groups=0, K=24, prefix=0, own=9000, queries=63, hq=16, hk=2, D=64, page=32),
        # a small fp32 policy
        dict(name="tree-f32", kind="tree", dtype="f32", groups=3, K=4, prefix=300, own=61, queries=13, hq=8, hk=2, D=64, page=16),
        # the next token of the 4 candidates of one turn, with all penalties: latency
        dict(name="rules-turn", kind="rules", dtype="bf16", V=151936, groups=1, K=4, prompt=197, own=32, queries=1, penalties=True, biases=0,
             masks=0, out=True),
        # drafted tokens of up to 128 candidates, each behind its own path, with biases and a grammar besides
        dict(name="rules-tree", kind="rules", dtype="bf16", V=151936, groups=16, K=8, prompt=1200, own=300, queries=8, penalties=True, biases=100,
             masks=40, out=True),
        # up to 1536 candidates under a grammar of 200 states: the best token that it allows and its probability, no logits
        dict(name="rules-grammar", kind="rules", dtype="bf16", V=151936, groups=192, K=8, prompt=600, own=64, queries=1, penalties=False, biases=0,
             masks=200, out=False),
        # an odd vocabulary in fp32
        dict(name="rules-f32", kind="rules", dtype="f32", V=32003, groups=11, K=4, prompt=300, own=200, queries=3, penalties=True, biases=17,
             masks=5, out=True),
    ]


# ---- cases of the same ranges --------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["plan", "tree", "tree", "rules", "rules"])
    if kind == "plan":
        page = rng.choice([8, 16, 32, 64])
        if rng.random() < 0.3:
            add = _log(rng, 16, 1100)
            return dict(kind=kind, groups=0, K=_log(rng, 1, min(2000, 380000 // add)), prefix=0, held=0, add=add, page=page, keep="all", tree=False)
        tree = rng.random() < 0.6
        return dict(kind=kind, groups=_log(rng, 1, 400), K=rng.choice([2, 4, 8]), prefix=_log(rng, 16, 1000), held=_log(rng, 8, 1500),
                    add=rng.randint(2, 40) if tree else 1, page=page, keep=rng.choice(["all", "some"]), tree=tree)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "rules":
        V = rng.choice([2048, _log(rng, 500, 151936), 151936])
        queries = rng.choice([1, 1, rng.randint(2, 16)])
        K = rng.choice([2, 4, 8])
        out = rng.random() < 0.7
        rows = min(1300, 190_000_000 // V // (4 if dtype == "f32" else 2))
        penalties, masks = rng.random() < 0.7, _log(rng, 1, 200) if rng.random() < 0.6 else 0
        return dict(kind=kind, dtype=dtype, V=V, groups=_log(rng, 1, max(1, rows // (K * queries))), K=K, prompt=_log(rng, 16, 2000), own=_log(rng, 8, 1000),
                    queries=queries, penalties=penalties or not masks, biases=rng.choice([0, _log(rng, 1, min(300, V // 2))]), masks=masks, out=out)
    hk = rng.choice([1, 2, 4, 8])
    c = dict(kind=kind, dtype=dtype, hk=hk, hq=hk * rng.choice([1, 2, 3, 4, 8] if hk < 8 else [1, 2, 4]), D=rng.choice([64, 128, 128]),
             page=rng.choice([16, 16, 32, 64]))
    queries = rng.choice([rng.randint(2, 8), rng.randint(4, 24), rng.randint(16, 64)])
    most = 180_000_000 // (c["hq"] * (8 if dtype == "f32" else 1))      # pairs of a query with a token, by what their products cost
    if rng.random() < 0.3:
        own_ = _log(rng, max(64, queries), 9000)
        return dict(c, groups=0, K=max(1, min(_log(rng, 1, 32), most // (own_ * queries))), prefix=0, own=own_, queries=queries)
    prefix, own_, K = _log(rng, 32, 40000), _log(rng, max(8, queries), 1500), rng.choice([2, 4, 8])
    queries = max(2, min(queries, most // (K * (prefix + own_))))
    seqs = max(K, min(256, 400000 // (prefix + own_), most // ((prefix + own_) * queries)))
    return dict(c, groups=max(1, min(32, _log(rng, 1, 32), seqs // K)), K=K, prefix=prefix, own=own_, queries=queries)


# ---- what a program holds before the call ----------------------------------------------------------
def _numbers(case):
    return np.random.default_rng([case["groups"], case["K"], 7 + sum(map(ord, case["kind"])), case.get("queries", case.get("add"))])


def _groups(case, rs, prompt):
    """Candidates of each group and their prompts' lengths."""
    G, K = case["groups"], case["K"]
    if not G:
        return np.array([K]), np.array([0])
    size, prefix = rs.integers(max(1, K - K // 4), K + 1, G), rs.integers(max(1, prompt // 3), prompt + 1, G)
    size[0], prefix[0] = K, prompt
    return size, prefix


def _parents(rs, new):
    """Trees: the first token of each is the root, every other one hangs on one of the eight in front of it; for each its number in its tree."""
    start = np.concatenate([[0], np.cumsum(new)])
    j = np.arange(start[-1]) - np.repeat(start[:-1], new)
    back = 1 + (rs.random(len(j)) * np.minimum(j, 8)).astype(np.int64)
    return np.where(j == 0, -1, j - back), j, start


def _ancestors(parent, start):
    """Bits of the tokens on the way from each to its root, itself among them."""
    bits = np.zeros(len(parent), np.uint64)
    for s in range(len(start) - 1):
        for t in range(start[s], start[s + 1]):
            bits[t] = np.uint64(1 << (t - start[s])) | (bits[start[s] + parent[t]] if parent[t] >= 0 else np.uint64(0))
    return bits.view(np.int64)


def _lognormal(rs, most, n):
    return np.clip(np.exp(rs.normal(math.log(max(1.0, most / 5.0)), 0.6, n)), 1, most).astype(np.int64)


def _sequences(case, seed):
    """Candidates of each group, prompts' lengths, the sequences' own tokens (those of the tree counted), tokens of their trees, and the
    trees.  A case has the same lengths under every seed, and therefore the same work, in an order that goes by the seed."""
    rs, order = _numbers(case), np.random.default_rng([seed, 77])
    size, prefix = _groups(case, rs, case["prefix"] if "prefix" in case else case["prompt"])
    if case["groups"]:
        size, prefix = order.permutation(size), order.permutation(prefix)
    n = int(size.sum())
    most, q = case["own"], case["queries"]
    length = rs.integers(max(1, most // 3), most + 1, n) if not case["groups"] else _lognormal(rs, most, n)
    length[-1] = most
    new = np.minimum(length, rs.integers((q + 1) // 2, q + 1, n))
    new[-1] = min(q, most)
    which = order.permutation(n)
    length, new = length[which], new[which]
    return size, prefix, length, new, *_parents(np.random.default_rng([seed, 78]), new)


def _pages_of(case, seed):
    """For a plan: tokens held, kept and added."""
    rs, order = _numbers(case), np.random.default_rng([seed, 77])
    size, prefix = _groups(case, rs, case["prefix"])
    if case["groups"]:
        size, prefix = order.permutation(size), order.permutation(prefix)
    n, most = int(size.sum()), case["add"]
    held = _lognormal(rs, case["held"], n) if case["held"] else np.zeros(n, np.int64)
    if most <= 64:
        add = rs.integers((most + 1) // 2, most + 1, n)
    else:
        add = rs.integers(max(1, most // 3), most + 1, n)
        add[0] = most
    keep = held.copy()
    if case["keep"] == "some":
        keep = np.maximum(0, held - rs.integers(0, 13, n))
        ended = rs.random(n) < 0.06
        keep, add = np.where(ended, 0, keep), np.where(ended, 0, add)
    which = order.permutation(n)
    return size, prefix, held[which], keep[which], add[which]


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt = torch.bfloat16 if case.get("dtype") == "bf16" else torch.float32

    def i32(a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(dev)

    def starts(a):
        return i32(np.concatenate([[0], np.cumsum(a)]))

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=gen, device=dev) * scale).to(dt)

    def table(used, ids):
        """Pages `ids`, as many for each row as it uses."""
        out = np.zeros((len(used), max(1, int(used.max(initial=0)))), np.int32)
        out[np.arange(out.shape[1])[None] < used[:, None]] = ids[:int(used.sum())]
        return out

    G = case["groups"]
    if case["kind"] == "plan":
        page = case["page"]
        size, prefix, held, keep, add = _pages_of(case, seed)
        used, will = -(-held // page), -(-(keep + add) // page)
        n_pages = int(np.maximum(used, will).sum()) + 5
        rs = np.random.default_rng([seed, 79])
        ids = rs.permutation(n_pages).astype(np.int32)
        pages = np.zeros((len(held), int(max(used.max(), will.max())) + 1), np.int32)
        pages[:, :max(1, int(used.max(initial=0)))] = table(used, ids)
        free = ids[int(used.sum()):]
        first = int(rs.integers(0, n_pages))
        ring = np.zeros(n_pages, np.int32)
        ring[(first + np.arange(len(free))) % n_pages] = free
        st = dict(case=case, length=i32(held), add=i32(add), keep=None if case["keep"] == "all" else i32(keep), pages=i32(pages), ring=i32(ring),
                  state=i32([first, len(free)]), n_tok=int(add.sum()), parent=None,
                  group_seq=starts(size) if G else None, prefix_len=i32(prefix) if G else None)
        if case["tree"]:
            st["parent"] = i32(_parents(np.random.default_rng([seed, 78]), add)[0])
        return st

    size, prefix, length, new, parent, j, start = _sequences(case, seed)
    bits = torch.from_numpy(_ancestors(parent, start)).to(dev)
    n_seq, n_tok = len(length), int(start[-1])
    st = dict(case=case, n_seq=n_seq, n_tok=n_tok, max_q=int(new.max()), ancestors=bits, length=i32(length),
              group_seq=starts(size) if G else None, prefix_len=i32(prefix) if G else None)
    if case["kind"] == "tree":
        page, hq, hk, D = case["page"], case["hq"], case["hk"], case["D"]
        used, shared = -(-length // page), -(-prefix // page)
        n_pages = int(used.sum()) + (int(shared.sum()) if G else 0) + 3
        ids = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32).cpu().numpy()      # pages lie anywhere
        st.update(cache_k=normal(n_pages, hk, page, D), cache_v=normal(n_pages, hk, page, D), pages=i32(table(used, ids)),
                  prefix_pages=i32(table(shared, ids[int(used.sum()):])) if G else None, cu_q=starts(new), q=normal(n_tok, hq, D, scale=1.5),
                  most=int(prefix.max()) + int(length.max()))
        return st

    V = case["V"]
    single = case["queries"] == 1
    # tokens of text: few are frequent
    words = torch.randperm(V, generator=gen, device=dev).to(torch.int32)

    def text(*shape):
        return words[(torch.rand(*shape, generator=gen, device=dev) ** 3 * V).long().clamp(max=V - 1)]

    # the drafted tokens are not yet among a sequence's own
    st.update(length=i32(length - (0 if single else new)), cu_q=None if single else starts(new), tokens=text(n_seq, case["own"]),
              prompt=text(G, int(prefix.max())) if G else None, logits=normal(n_tok, V, scale=2.5))
    if single:
        st["ancestors"] = None
    st["drafted"] = None if single else text(n_tok)
    uniform = lambda lo, hi: lo + (hi - lo) * torch.rand(n_seq, generator=gen, device=dev)
    st.update({name: uniform(lo, hi) if case["penalties"] else None for name, lo, hi in
               (("repetition", 1.0, 1.4), ("presence", 0.0, 0.5), ("frequency", 0.0, 0.3), ("temperature", 0.6, 1.2))})
    st.update(bias_cu=None, bias_token=None, bias=None, mask_row=None, allowed=None)
    if case["biases"]:
        rs = np.random.default_rng([seed, 80])
        count = rs.integers(case["biases"] // 2, case["biases"] + 1, n_seq)
        st.update(bias_cu=starts(count), bias_token=i32(np.concatenate([rs.choice(V, c, replace=False) for c in count])),
                  bias=torch.randn(int(count.sum()), generator=gen, device=dev) * 4)
    if case["masks"]:
        words_of = -(-V // 32)
        allowed = torch.zeros(case["masks"], words_of, dtype=torch.int32, device=dev)
        for m in range(case["masks"]):      # states allow few tokens, or most
            share = (0.0005, 0.02, 0.3, 0.95)[m % 4]
            bit = torch.rand(words_of, 32, generator=gen, device=dev) < share
            value = (bit.long() << torch.arange(32, device=dev)).sum(1)
            allowed[m] = torch.where(value >= 1 << 31, value - (1 << 32), value).to(torch.int32)
        st.update(allowed=allowed, mask_row=torch.randint(-1, case["masks"], (n_tok,), generator=gen, device=dev, dtype=torch.int32))
    return st


# ---- one pass ---------------------------------------------------------------------------------------
def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    from paper_2510_11062_amd import api
    kind = st["case"]["kind"]
    if kind == "plan":
        pool = api.PagePool(st["pages"], st["ring"], st["case"]["page"], group_seq=st["group_seq"], prefix_len=st["prefix_len"])
        o = api.at_grpo_kv_plan(pool, st["length"], st["add"], st["state"], st["n_tok"], keep=st["keep"], parent=st["parent"])
        out = {n: o[n] for n in ("length", "state", "cu_q", "seq", "position", "slot")}
        out.update(pages=st["pages"], ring=st["ring"])
        if st["parent"] is not None:
            out["ancestors"] = o["ancestors"]
        return out
    if kind == "tree":
        kv = api.KVBatch(st["cache_k"], st["cache_v"], st["pages"], st["length"], cu_q=st["cu_q"], group_seq=st["group_seq"],
                         prefix_len=st["prefix_len"], prefix_pages=st["prefix_pages"])
        return {"out": api.at_grpo_tree_attention(kv, st["q"], st["ancestors"], max_q=st["max_q"])["out"]}
    rules = api.LogitRules(tokens=st["tokens"], length=st["length"], prompt=st["prompt"], prompt_len=st["prefix_len"], group_seq=st["group_seq"],
                           cu_q=st["cu_q"], drafted=st["drafted"], ancestors=st["ancestors"], repetition=st["repetition"], presence=st["presence"],
                           frequency=st["frequency"], temperature=st["temperature"], bias_cu=st["bias_cu"], bias_token=st["bias_token"],
                           bias=st["bias"], allowed=st["allowed"], mask_row=st["mask_row"])
    o = api.at_grpo_logit_rules(rules, st["logits"], want_out=st["case"]["out"])
    return {n: o[n] for n in (("out",) if st["case"]["out"] else ()) + ("lse", "best")}


def _run_plain(st):
    return {"plan": _plain_plan, "tree": _plain_tree, "rules": _plain_rules}[st["case"]["kind"]](st)


def _before(x):
    return torch.cat((torch.zeros(1, dtype=x.dtype, device=x.device), x.cumsum(0)))


def _prefixes(st, n_seq):
    """For each sequence its group and its prompt's length."""
    dev = st["length"].device
    if st["group_seq"] is None:
        return None, torch.zeros(n_seq, dtype=torch.int64, device=dev)
    group = torch.searchsorted(st["group_seq"].long(), torch.arange(n_seq, device=dev), right=True) - 1
    return group, st["prefix_len"].long()[group]


def _plain_plan(st):
    page, n_tok, dev = st["case"]["page"], st["n_tok"], st["length"].device
    held, add, ring, pages = st["length"].long(), st["add"].long(), st["ring"], st["pages"]
    keep = held if st["keep"] is None else st["keep"].long()
    n_seq, n_pages = len(held), len(ring)
    used, will = (held + page - 1) // page, (keep + add + page - 1) // page
    take, give = (will - used).clamp(min=0), (used - will).clamp(min=0)
    first, count = st["state"].long().unbind()
    col = torch.arange(pages.shape[1], device=dev)[None]
    from_ring = (first + _before(take)[:-1, None] + col - used[:, None]) % n_pages
    new_pages = torch.where((col >= used[:, None]) & (col < will[:, None]), ring[from_ring], pages)
    to_ring = (first + count + _before(give)[:-1, None] + col - will[:, None]) % n_pages
    to_ring = torch.where((col >= will[:, None]) & (col < used[:, None]), to_ring, n_pages)
    new_ring = torch.cat((ring, ring[:1])).scatter(0, to_ring.flatten(), pages.flatten())[:n_pages]
    state = torch.stack(((first + take.sum()) % n_pages, count - take.sum() + give.sum()))
    cu = _before(add)
    token = torch.arange(n_tok, device=dev)
    seq = torch.searchsorted(cu, token, right=True) - 1
    j = token - cu[seq]
    place = keep[seq] + j
    slot = new_pages[seq, place // page].long() * page + place % page
    i32 = torch.int32
    out = dict(length=(keep + add).to(i32), state=state.to(i32), cu_q=cu.to(i32), seq=seq.to(i32), slot=slot, pages=new_pages, ring=new_ring)
    depth = j
    if st["parent"] is not None:
        bits, up = torch.ones_like(j) << j, torch.where(st["parent"] < 0, -1, cu[seq] + st["parent"].long())
        for _ in range(6):      # each time twice as far
            bits = torch.where(up < 0, bits, bits | bits[up.clamp(min=0)])
            up = torch.where(up < 0, -1, up[up.clamp(min=0)])
        out["ancestors"] = bits
        depth = ((bits[:, None] >> torch.arange(64, device=dev)) & 1).sum(1) - 1
    out["position"] = (_prefixes(st, n_seq)[1][seq] + keep[seq] + depth).to(i32)
    return out


def _plain_tree(st):
    case, dev, n_seq, Q, L = st["case"], st["q"].device, st["n_seq"], st["max_q"], st["most"]
    page, hq, hk, D = case["page"], case["hq"], case["hk"], case["D"]
    cu = st["cu_q"].long()
    new = cu[1:] - cu[:-1]
    group, prefix = _prefixes(st, n_seq)
    at = torch.arange(L, device=dev)[None]
    in_own = at - prefix[:, None]                                     # [n_seq, L], negative inside the prompt
    where = st["pages"].long().gather(1, (in_own.clamp(min=0) // page).clamp(max=st["pages"].shape[1] - 1))
    offset = in_own.clamp(min=0) % page
    if group is not None:
        shared = st["prefix_pages"].long()[group].gather(1, (at // page).clamp(max=st["prefix_pages"].shape[1] - 1).expand(n_seq, L))
        where, offset = torch.where(in_own < 0, shared, where), torch.where(in_own < 0, at % page, offset)
    k = st["cache_k"][where, :, offset].float().permute(0, 2, 3, 1)    # [n_seq, hk, D, L]
    v = st["cache_v"][where, :, offset].float().permute(0, 2, 1, 3)    # [n_seq, hk, L, D]
    j = torch.arange(Q, device=dev)[None]
    rows = (cu[:-1, None] + j).clamp(max=st["n_tok"] - 1)              # [n_seq, Q]
    q = st["q"][rows].float().view(n_seq, Q, hk, hq // hk, D).permute(0, 2, 1, 3, 4).reshape(n_seq, hk, Q * (hq // hk), D)
    z = (q @ k).view(n_seq, hk, Q, hq // hk, L) / math.sqrt(D)
    in_tree = (at - (prefix + st["length"].long() - new)[:, None])[:, None]          # [n_seq, 1, L]
    sees = (in_tree < 0) | ((in_tree < new[:, None, None]) & ((st["ancestors"][rows][..., None] >> in_tree.clamp(0, 63)) & 1).bool())
    z = z.masked_fill(~sees[:, None, :, None], -math.inf)
    e = torch.exp(z - z.amax(-1, keepdim=True))
    o = (e.view(n_seq, hk, -1, L) @ v).view(n_seq, hk, Q, hq // hk, D) / e.sum(-1, keepdim=True)
    o = o.permute(0, 2, 1, 3, 4).reshape(n_seq, Q, hq, D)
    seq = torch.searchsorted(cu, torch.arange(st["n_tok"], device=dev), right=True) - 1
    return {"out": o[seq, torch.arange(st["n_tok"], device=dev) - cu[seq]].to(st["q"].dtype)}


def _plain_rules(st):
    logits, dev = st["logits"], st["logits"].device
    n, V = logits.shape
    row = torch.arange(n, device=dev)
    seq = row if st["cu_q"] is None else torch.searchsorted(st["cu_q"].long(), row, right=True) - 1
    z = logits.float()
    if st["repetition"] is not None:
        of = lambda name: st[name][seq][:, None]
        own_ = st["tokens"].long()[seq]
        there = torch.arange(own_.shape[1], device=dev) < st["length"][seq][:, None]
        count = torch.zeros(n, V, device=dev).scatter_add_(1, own_, there.float())
        if st["ancestors"] is not None:
            bit = torch.arange(64, device=dev)
            path = st["drafted"].long()[(st["cu_q"].long()[seq][:, None] + bit).clamp(max=n - 1)]
            count.scatter_add_(1, path, ((st["ancestors"][:, None] >> bit) & 1).float())
        seen = count > 0
        if st["prompt"] is not None:
            group, size = _prefixes(st, st["n_seq"])
            prompt = st["prompt"].long()[group[seq]]
            there = torch.arange(prompt.shape[1], device=dev) < size[seq][:, None]
            seen |= torch.zeros(n, V, device=dev).scatter_add_(1, prompt, there.float()) > 0
        z = torch.where(seen, torch.where(z > 0, z / of("repetition"), z * of("repetition")), z)
        z = torch.where(count > 0, z - of("frequency") * count - of("presence"), z)
    if st["bias"] is not None:
        entry = torch.searchsorted(st["bias_cu"].long(), torch.arange(len(st["bias"]), device=dev), right=True) - 1
        z = z + torch.zeros(st["n_seq"], V, device=dev).index_put((entry, st["bias_token"].long()), st["bias"])[seq]
    if st["allowed"] is not None:
        v = torch.arange(V, device=dev)
        ok = (st["allowed"][st["mask_row"].clamp(min=0).long()][:, v // 32] >> (v % 32)) & 1
        z = z.masked_fill((ok == 0) & (st["mask_row"] >= 0)[:, None], -math.inf)
    top = z.amax(1, keepdim=True)
    best = torch.where((z == top) & (z > -math.inf), torch.arange(V, device=dev, dtype=torch.int32), V).amin(1)
    best = torch.where(best == V, -1, best).to(torch.int32)
    if st["temperature"] is not None:
        f = (1.0 / st["temperature"][seq])[:, None]
        z, top = z * f, top * f
    lse = torch.log(torch.exp(z - torch.where(top > -math.inf, top, 0.0)).sum(1)) + top[:, 0]
    out = {"lse": lse, "best": best}
    if st["case"]["out"]:
        out["out"] = z.to(logits.dtype)
    return out


# ---- what a pass cannot do without ------------------------------------------------------------------
def work(case):
    if case["kind"] == "plan":
        size, prefix, held, keep, add = _pages_of(case, 0)
        moved, n = int(np.abs(-(-(keep + add) // case["page"]) - -(-held // case["page"])).sum()), int(add.sum())
        tokens = n * (16 + (12 if case["tree"] else 0))
        return {"bytes": len(held) * (16 if case["keep"] == "all" else 20) + 8 * len(prefix) + 8 * moved + tokens, "flops": 10 * n}
    e = 2 if case["dtype"] == "bf16" else 4
    size, prefix, length, new, parent, j, start = _sequences(case, 0)
    n, prompts = int(new.sum()), int(prefix.sum()) if case["groups"] else 0
    if case["kind"] == "tree":
        hq, hk, D = case["hq"], case["hk"], case["D"]
        bits = _ancestors(parent, start).view(np.uint8).reshape(n, 8)
        seen = int((new * (np.repeat(prefix, size) + length - new)).sum()) + int(np.unpackbits(bits, axis=1).sum())
        return {"bytes": 2 * (prompts + int(length.sum())) * hk * D * e + 2 * n * hq * D * e + 8 * n, "flops": 4 * seen * hq * D}
    V = case["V"]
    lists = 4 * (prompts + int(length.sum())) + 16 * len(length) if case["penalties"] else 0
    lists += 6 * case["biases"] * len(length) + (4 * n + case["masks"] * V // 8 if case["masks"] else 0)
    return {"bytes": n * V * e * (2 if case["out"] else 1) + lists + 8 * n + (0 if case["queries"] == 1 else 12 * n), "flops": 6 * n * V}


# ---- the definitions in 64 bits ---------------------------------------------------------------------
def exact(case, seed):
    return {"plan": _exact_plan, "tree": _exact_tree, "rules": _exact_rules}[case["kind"]](case, seed)


def _exact_plan(case, seed):
    st, page = prepare(case, seed), case["page"]
    host = lambda name: st[name].cpu().numpy().astype(np.int64)
    size, prefix, held, keep, add = _pages_of(case, seed)
    ring, pages = host("ring"), host("pages")
    (first, count), group = host("state"), np.repeat(np.arange(len(size)), size)
    parent = None if st["parent"] is None else host("parent")
    tail = first + count
    out = dict(length=keep + add, cu_q=[0], seq=[], position=[], slot=[], ancestors=[])
    for s in range(len(held)):
        have, want = -(-held[s] // page), -(-(keep[s] + add[s]) // page)
        for i in range(have, want):
            pages[s, i] = ring[first % len(ring)]
            first, count = first + 1, count - 1
        for i in range(want, have):
            ring[tail % len(ring)] = pages[s, i]
            tail, count = tail + 1, count + 1
        paths = []
        for j in range(int(add[s])):
            path = {j}
            if parent is not None and parent[out["cu_q"][-1] + j] >= 0:
                path |= paths[parent[out["cu_q"][-1] + j]]
            paths.append(path if parent is not None else None)
            place = int(keep[s]) + j
            out["seq"].append(s)
            out["slot"].append(int(pages[s, place // page]) * page + place % page)
            out["position"].append(int(prefix[group[s]]) + int(keep[s]) + (len(path) - 1 if parent is not None else j))
            if parent is not None:
                out["ancestors"].append(sum(1 << i for i in path))
        out["cu_q"].append(out["cu_q"][-1] + int(add[s]))
    out.update(pages=pages, ring=ring, state=[first % len(ring), count])
    if parent is None:
        del out["ancestors"]
    return {n: torch.from_numpy(np.array(x, np.uint64 if n == "ancestors" else np.int64).view(np.int64)) for n, x in out.items()}


def _exact_tree(case, seed):
    st = prepare(case, seed)
    page, hq, hk, D, dev = case["page"], case["hq"], case["hk"], case["D"], st["q"].device
    size, prefix, length, new, parent, j, start = _sequences(case, seed)
    group = np.repeat(np.arange(len(size)), size)
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=dev)

    def rows(cache, table, n):
        at = torch.arange(int(n), device=dev)
        return cache[table[at // page].long(), :, at % page].double()          # [n, hk, D]

    last = None
    for s in range(len(length)):
        g, m, t0 = int(group[s]), int(new[s]), int(start[s])
        k, v = (rows(st[c], st["pages"][s], length[s]) for c in ("cache_k", "cache_v"))
        if case["groups"]:
            if last is None or last[0] != g:
                last = (g, *(rows(st[c], st["prefix_pages"][g], prefix[g]) for c in ("cache_k", "cache_v")))
            k, v = torch.cat((last[1], k)), torch.cat((last[2], v))
        tree = np.zeros((m, m), bool)
        for i in range(m):
            at = i
            while at >= 0:
                tree[i, at] = True
                at = int(parent[t0 + at])
        sees = torch.ones(m, k.shape[0], dtype=torch.bool, device=dev)
        sees[:, k.shape[0] - m:] = torch.from_numpy(tree).to(dev)
        q = st["q"][t0:t0 + m].double().view(m, hk, hq // hk, D)
        for h in range(hk):
            z = (q[:, h].reshape(-1, D) @ k[:, h].T).view(m, hq // hk, -1) / math.sqrt(D)
            p = torch.softmax(z.masked_fill(~sees[:, None], -math.inf), -1)
            out[t0:t0 + m, h * (hq // hk):(h + 1) * (hq // hk)] = (p.view(m * (hq // hk), -1) @ v[:, h]).view(m, -1, D)
    return {"out": out}


def _exact_rules(case, seed):
    st = prepare(case, seed)
    size, prefix, length, new, parent, j, start = _sequences(case, seed)
    n, V = st["logits"].shape
    dev, group = st["logits"].device, np.repeat(np.arange(len(size)), size)
    lse = torch.empty(n, dtype=torch.float64, device=dev)
    best = torch.empty(n, dtype=torch.int64, device=dev)
    out = torch.empty(n, V, dtype=torch.float64, device=dev) if case["out"] else None
    mask_row = [-1] * n if st["mask_row"] is None else st["mask_row"].tolist()
    bias_cu = None if st["bias_cu"] is None else st["bias_cu"].tolist()
    setting = {x: [1.0 if x in ("repetition", "temperature") else 0.0] * len(length) if st[x] is None else st[x].double().tolist()
               for x in ("repetition", "presence", "frequency", "temperature")}
    bits = torch.arange(32, device=dev)
    single = st["cu_q"] is None
    for s in range(len(length)):
        own_ = st["tokens"][s, :int(length[s]) - (0 if single else int(new[s]))].long()
        for t in range(s, s + 1) if single else range(int(start[s]), int(start[s + 1])):
            z = st["logits"][t].double()
            if case["penalties"]:
                path, at = own_, -1 if single else t - int(start[s])
                while at >= 0:
                    path = torch.cat((path, st["drafted"][int(start[s]) + at].long()[None]))
                    at = int(parent[int(start[s]) + at])
                count = torch.bincount(path, minlength=V)
                seen = count > 0
                if case["groups"]:
                    seen = seen | (torch.bincount(st["prompt"][int(group[s]), :int(prefix[group[s]])].long(), minlength=V) > 0)
                r = setting["repetition"][s]
                z = torch.where(seen, torch.where(z > 0, z / r, z * r), z)
                z = z - setting["frequency"][s] * count - setting["presence"][s] * (count > 0)
            if bias_cu is not None:
                e = slice(bias_cu[s], bias_cu[s + 1])
                z[st["bias_token"][e].long()] += st["bias"][e].double()
            if mask_row[t] >= 0:
                ok = ((st["allowed"][mask_row[t]][:, None] >> bits) & 1).bool().flatten()[:V]
                z = z.masked_fill(~ok, -math.inf)
            best[t] = torch.where(z == z.max(), torch.arange(V, device=dev), V).min()
            if bool((z == -math.inf).all()):
                best[t] = -1
            z = z / setting["temperature"][s]
            lse[t] = torch.logsumexp(z, 0)
            if out is not None:
                out[t] = z
    return {"out": out, "lse": lse, "best": best} if case["out"] else {"lse": lse, "best": best}
