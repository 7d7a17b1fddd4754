"""The operators in front of the policy loss, as cases that can be timed and compared: queries and keys normed and rotated
(forward and gradient), appended to a paged cache, and attention of candidates that share a prompt.

A case is a dict of plain values; `prepare` builds on the GPU what a rollout or training program holds before the call, `run` is
one pass, through the library's entry points where `own` is true and in elementary torch operations where it is not.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

EPS = 1e-6


def listed():
    return [
        # training, the rows of a single response of 197 tokens: latency
        dict(name="rotate-response", kind="rotate", dtype="bf16", n=197, hq=16, hk=8, D=128, rot=128, interleaved=False),
        # training, a micro-batch of 16384 rows of a policy with H = 4096
        dict(name="rotate-batch", kind="rotate", dtype="bf16", n=16384, hq=32, hk=8, D=128, rot=128, interleaved=False),
        # the gradient for as many rows of a policy with H = 2048, an odd number
        dict(name="rotate-grad", kind="rotate_grad", dtype="bf16", n=16383, hq=16, hk=8, D=128, rot=128, interleaved=False),
        # the gradient of a small fp32 policy that rotates half of each head, pairs side by side
        dict(name="rotate-grad-f32", kind="rotate_grad", dtype="f32", n=3001, hq=8, hk=8, D=64, rot=32, interleaved=True),
        # one token for each of the 4 candidates of one turn: latency
        dict(name="append-turn", kind="append", dtype="bf16", groups=1, K=4, prefix=197, own=32, queries=1, hq=16, hk=8, D=128, rot=128,
             interleaved=False, page=16),
        # one token for each of up to 1536 candidates (C3's number of responses)
        dict(name="append-rollout", kind="append", dtype="bf16", groups=192, K=8, prefix=600, own=64, queries=1, hq=32, hk=8, D=128,
             rot=128, interleaved=False, page=16),
        # 64 prompts of up to 1100 tokens go into the cache, pairs side by side, a quarter of each head is not rotated
        dict(name="append-prompts", kind="append", dtype="bf16", groups=0, K=64, prefix=0, own=1100, queries=1100, hq=16, hk=8, D=128,
             rot=96, interleaved=True, page=64),
        # one token for each of the 4 candidates of one turn, a short prompt: latency
        dict(name="attend-turn", kind="attend", dtype="bf16", groups=1, K=4, prefix=197, own=32, queries=1, hq=16, hk=8, D=128, page=16),
        # tree sampling: 32 prompts of up to 2400 tokens, up to 8 candidates of each, responses of lognormal lengths
        dict(name="attend-tree", kind="attend", dtype="bf16", groups=32, K=8, prefix=2400, own=1500, queries=1, hq=32, hk=8, D=128, page=16),
        # two long prompts (a history of many turns), 8 candidates of each
        dict(name="attend-long", kind="attend", dtype="bf16", groups=2, K=8, prefix=40000, own=512, queries=1, hq=16, hk=8, D=128, page=64),
        # prompts of up to 2048 tokens attend to themselves, no prefix
        dict(name="attend-prompts", kind="attend", dtype="bf16", groups=0, K=8, prefix=0, own=2048, queries=2048, hq=16, hk=8, D=128, page=64),
        # fp32, the few tokens of another agent's message behind each candidate's own
        dict(name="attend-message-f32", kind="attend", dtype="f32", groups=3, K=4, prefix=300, own=61, queries=37, hq=8, hk=2, D=64, page=16),
    ]


# ---- cases of the same ranges --------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    hk = rng.choice([1, 2, 4, 8])
    return dict(hk=hk, hq=hk * rng.choice([1, 2, 3, 4, 8] if hk < 8 else [1, 2, 4]))


def draw(rng):
    kind = rng.choice(["rotate", "rotate_grad", "append", "append", "attend", "attend", "attend"])
    D = rng.choice([64, 128, 128])
    c = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]), D=D, **_heads(rng))
    if kind != "attend":
        c.update(rot=rng.choice([D, D, D // 2, 3 * D // 4]), interleaved=rng.random() < 0.4)
    if kind in ("rotate", "rotate_grad"):
        most = 16383 * 24 * 128 // ((c["hq"] + c["hk"]) * D * (2 if c["dtype"] == "f32" else 1))
        return dict(c, n=_log(rng, 64, min(16384, most)))
    c["page"] = rng.choice([16, 16, 32, 64])
    if kind == "append":
        if rng.random() < 0.6:
            groups, K = _log(rng, 1, 192), rng.choice([2, 4, 8])
            return dict(c, groups=groups, K=K, prefix=_log(rng, 16, 1000), own=_log(rng, 4, 64), queries=1)
        own_ = _log(rng, 16, 1100)
        return dict(c, groups=0, K=min(64, max(1, 24000 // own_)), prefix=0, own=own_, queries=own_)
    shape = rng.choice(["decode", "decode", "decode", "message", "prompts"])
    if shape == "prompts":
        own_ = _log(rng, 64, 1800 if c["dtype"] == "bf16" else 700)
        return dict(c, groups=0, K=max(1, min(8, _log(rng, 2, 8), 16 * 8 // c["hq"])), prefix=0, own=own_, queries=own_)
    prefix = _log(rng, 32, 40000)
    K = rng.choice([2, 4, 8])
    own_ = _log(rng, 8, 1000)
    seqs = max(K, min(256, 400000 // (prefix + own_)))
    groups = max(1, min(32, _log(rng, 1, 32), seqs // K))
    queries = 1 if shape == "decode" else min(own_, rng.randint(2, 48), max(1, 400 // c["hq"]))
    return dict(c, groups=groups, K=K, prefix=prefix, own=own_, queries=queries)


# ---- what a program holds before the call ----------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _rope_table(n_pos, rot, dev, base=1e6):
    """cos and sin of position times frequency, as a program keeps them for all layers: fp32 [n_pos, rot / 2, 2]."""
    f = base ** (-torch.arange(0, rot, 2, device=dev, dtype=torch.float64) / rot)
    a = torch.arange(n_pos, device=dev, dtype=torch.float64)[:, None] * f
    return torch.stack((a.cos(), a.sin()), -1).float()


def _plan(case, seed):
    """Host arrays: candidates of each group, prompt lengths, tokens in the cache of each sequence, new ones among them.  A case has
    the same lengths under every seed, and therefore the same work, in an order that goes by the seed."""
    G, K, most = case["groups"], case["K"], case["own"]
    rs = np.random.default_rng([G, K, most, case["prefix"], case["queries"]])
    order = np.random.default_rng([seed, 77])
    size, prefix = np.array([K]), np.array([0])
    if G:
        size = rs.integers(max(1, K - K // 4), K + 1, G)
        size[0] = K
        prefix = rs.integers(max(1, case["prefix"] // 3), case["prefix"] + 1, G)
        prefix[0] = case["prefix"]
        size, prefix = order.permutation(size), order.permutation(prefix)
    n_seq = int(size.sum())
    if case["queries"] == most:         # prompts: every token is new
        length = rs.integers(max(1, most // 3), most + 1, n_seq)
        length[0] = most
        new = length
    else:
        length = np.clip(np.exp(rs.normal(math.log(max(1.0, most / 5.0)), 0.6, n_seq)), 1, most).astype(np.int64)
        length[-1] = most
        new = np.minimum(length, rs.integers(1, case["queries"] + 1, n_seq))
        new[-1] = case["queries"]
    which = order.permutation(n_seq)
    return size, prefix, length[which], new[which]


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt = _dtype(case)
    hq, hk, D = case["hq"], case["hk"], case["D"]

    def normal(*shape, scale=1.0, mean=0.0):
        return (torch.randn(*shape, generator=gen, device=dev) * scale + mean).to(dt)

    st = dict(case=case)
    if case["kind"] in ("rotate", "rotate_grad"):
        n = case["n"]
        qkv = normal(n, (hq + 2 * hk) * D, scale=2.0)        # the projections' output: queries, keys and values side by side
        st.update(q=qkv[:, :hq * D].view(n, hq, D), k=qkv[:, hq * D:(hq + hk) * D].view(n, hk, D))
        st["position"] = torch.randint(0, 4096, (n,), generator=gen, device=dev, dtype=torch.int32)
        st["rope"] = _rope_table(4096, case["rot"], dev)
        st.update(q_weight=normal(D, scale=0.2, mean=1.0), k_weight=normal(D, scale=0.2, mean=1.0))
        if case["kind"] == "rotate_grad":
            st.update(dq=normal(n, hq, D, scale=0.01), dk=normal(n, hk, D, scale=0.01))
        return st
    size, prefix, length, new = _plan(case, seed)
    G, n_seq, page = case["groups"], len(length), case["page"]
    n_tok = int(new.sum())

    def i32(a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(dev)

    max_pages = -(-int(length.max()) // page)
    max_prefix_pages = -(-int(prefix.max()) // page)
    used = [-(-int(x) // page) for x in length] + ([-(-int(x) // page) for x in prefix] if G else [])
    n_pages = sum(used) + 3
    order = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32).cpu().numpy()      # pages lie anywhere
    tables = np.zeros((n_seq, max_pages), np.int32), np.zeros((max(G, 1), max(max_prefix_pages, 1)), np.int32)
    at = 0
    for i, u in enumerate(used):
        t, row = (tables[0], i) if i < n_seq else (tables[1], i - n_seq)
        t[row, :u] = order[at:at + u]
        at += u
    st.update(cache_k=normal(n_pages, hk, page, D), cache_v=normal(n_pages, hk, page, D), pages=i32(tables[0]), length=i32(length),
              cu_q=None if case["queries"] == 1 else i32(np.concatenate([[0], np.cumsum(new)])),
              group_seq=i32(np.concatenate([[0], np.cumsum(size)])) if G else None,
              prefix_len=i32(prefix) if G else None, prefix_pages=i32(tables[1]) if G else None,
              n_seq=n_seq, n_tok=n_tok, max_q=int(new.max()), most=case["prefix"] + case["own"])
    if case["kind"] == "append":
        qkv = normal(n_tok, (hq + 2 * hk) * D, scale=2.0)
        st.update(q=qkv[:, :hq * D].view(n_tok, hq, D), k=qkv[:, hq * D:(hq + hk) * D].view(n_tok, hk, D),
                  v=qkv[:, (hq + hk) * D:].view(n_tok, hk, D))
        st["rope"] = _rope_table(st["most"], case["rot"], dev)
        st.update(q_weight=normal(D, scale=0.2, mean=1.0), k_weight=normal(D, scale=0.2, mean=1.0))
    else:
        st["q"] = normal(n_tok, hq, D, scale=1.5)
    return st


# ---- one pass ---------------------------------------------------------------------------------------
def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    from paper_2510_11062_amd import api
    case = st["case"]
    kind = case["kind"]
    if kind == "rotate":
        o = api.at_grpo_qk_norm_rope(st["q"], st["k"], st["rope"], st["position"], st["q_weight"], st["k_weight"], eps=EPS,
                                     interleaved=case["interleaved"])
        return {"q": o["q"], "k": o["k"]}
    if kind == "rotate_grad":
        o = api.at_grpo_qk_norm_rope_bwd(st["dq"], st["dk"], st["q"], st["k"], st["rope"], st["position"], st["q_weight"],
                                         st["k_weight"], eps=EPS, interleaved=case["interleaved"])
        return {n: o[n] for n in ("dq", "dk", "dq_weight", "dk_weight")}
    kv = api.KVBatch(st["cache_k"], st["cache_v"], st["pages"], st["length"], cu_q=st["cu_q"], group_seq=st["group_seq"],
                     prefix_len=st["prefix_len"], prefix_pages=st["prefix_pages"])
    if kind == "append":
        o = api.at_grpo_kv_append(kv, st["q"], st["k"], st["v"], st["rope"], st["q_weight"], st["k_weight"], eps=EPS,
                                  interleaved=case["interleaved"])
        return {"q": o["q"], "cache_k": st["cache_k"], "cache_v": st["cache_v"]}
    return {"out": api.at_grpo_prefix_attention(kv, st["q"], max_q=st["max_q"])["out"]}


def _pairs(x, r, interleaved):
    return (x[..., :r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])


def _unpair(a, b, rest, interleaved):
    both = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((both, rest), -1)


def _norm_rope(x, w, rope, position, interleaved):
    x = x.float()
    u = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    r = 2 * rope.shape[1]
    cs = rope[position.long()][:, None]
    c, s = cs[..., 0], cs[..., 1]
    a, b = _pairs(u, r, interleaved)
    return _unpair(a * c - b * s, b * c + a * s, u[..., r:], interleaved)


def _norm_rope_grad(dy, x, w, rope, position, interleaved):
    dy, x, w = dy.float(), x.float(), w.float()
    r = 2 * rope.shape[1]
    cs = rope[position.long()][:, None]
    c, s = cs[..., 0], cs[..., 1]
    a, b = _pairs(dy, r, interleaved)
    g = _unpair(a * c + b * s, b * c - a * s, dy[..., r:], interleaved)
    rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    xh = x * rstd
    gw = g * w
    return rstd * (gw - xh * (gw * xh).mean(-1, keepdim=True)), (g * xh).sum((0, 1))


def _places(st):
    """For each new token its sequence and its place in it; for each sequence its new tokens, where they begin, its group's prompt."""
    dev = st["length"].device
    seqs = torch.arange(st["n_seq"], device=dev)
    cu = torch.arange(st["n_seq"] + 1, device=dev) if st["cu_q"] is None else st["cu_q"].long()
    new = cu[1:] - cu[:-1]
    if st["group_seq"] is None:
        prefix, group = torch.zeros_like(seqs), None
    else:
        group = torch.searchsorted(st["group_seq"].long(), seqs, right=True) - 1
        prefix = st["prefix_len"].long()[group]
    tokens = torch.arange(st["n_tok"], device=dev)
    seq = torch.searchsorted(cu, tokens, right=True) - 1
    place = st["length"].long()[seq] - new[seq] + tokens - cu[seq]
    return seq, place, new, cu, prefix, group


def _run_plain(st):
    case = st["case"]
    kind, dt = case["kind"], _dtype(case)
    if kind == "rotate":
        return {"q": _norm_rope(st["q"], st["q_weight"], st["rope"], st["position"], case["interleaved"]).to(dt),
                "k": _norm_rope(st["k"], st["k_weight"], st["rope"], st["position"], case["interleaved"]).to(dt)}
    if kind == "rotate_grad":
        dq, dwq = _norm_rope_grad(st["dq"], st["q"], st["q_weight"], st["rope"], st["position"], case["interleaved"])
        dk, dwk = _norm_rope_grad(st["dk"], st["k"], st["k_weight"], st["rope"], st["position"], case["interleaved"])
        return {"dq": dq.to(dt), "dk": dk.to(dt), "dq_weight": dwq, "dk_weight": dwk}
    page, hq, hk, D = case["page"], case["hq"], case["hk"], case["D"]
    seq, place, new, cu, prefix, group = _places(st)
    if kind == "append":
        position = prefix[seq] + place
        q = _norm_rope(st["q"], st["q_weight"], st["rope"], position, case["interleaved"]).to(dt)
        k = _norm_rope(st["k"], st["k_weight"], st["rope"], position, case["interleaved"]).to(dt)
        where = st["pages"].long()[seq, place // page]
        st["cache_k"][where, :, place % page] = k
        st["cache_v"][where, :, place % page] = st["v"]
        return {"q": q, "cache_k": st["cache_k"], "cache_v": st["cache_v"]}
    n_seq, Q, L, dev = st["n_seq"], st["max_q"], st["most"], st["q"].device
    at = torch.arange(L, device=dev)[None]
    in_own = at - prefix[:, None]                                     # [n_seq, L], negative inside the prompt
    where = st["pages"].long().gather(1, (in_own.clamp(min=0) // page).clamp(max=st["pages"].shape[1] - 1))
    offset = in_own.clamp(min=0) % page
    if group is not None:
        table = st["prefix_pages"].long()[group]
        shared = table.gather(1, (at // page).clamp(max=table.shape[1] - 1).expand(n_seq, L))
        where, offset = torch.where(in_own < 0, shared, where), torch.where(in_own < 0, at % page, offset)
    k = st["cache_k"][where, :, offset].float().permute(0, 2, 3, 1)    # [n_seq, hk, D, L]
    v = st["cache_v"][where, :, offset].float().permute(0, 2, 1, 3)    # [n_seq, hk, L, D]
    j = torch.arange(Q, device=dev)[None]
    rows = (cu[:-1, None] + j).clamp(max=st["n_tok"] - 1)              # [n_seq, Q]
    q = st["q"][rows].float().view(n_seq, Q, hk, hq // hk, D).permute(0, 2, 1, 3, 4).reshape(n_seq, hk, Q * (hq // hk), D)
    z = (q @ k).view(n_seq, hk, Q, hq // hk, L) / math.sqrt(D)
    seen = (prefix + st["length"].long() - new)[:, None] + j            # the last place that a new token sees
    z = z.masked_fill((at[:, None] > seen[..., None])[:, None, :, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(torch.isfinite(top), top, 0.0))
    total = e.sum(-1, keepdim=True)
    o = (e.view(n_seq, hk, -1, L) @ v).view(n_seq, hk, Q, hq // hk, D) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 2, 1, 3, 4).reshape(n_seq, Q, hq, D)
    return {"out": o[seq, torch.arange(st["n_tok"], device=dev) - cu[seq]].to(dt)}


# ---- what a pass cannot do without ------------------------------------------------------------------
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    hq, hk, D = case["hq"], case["hk"], case["D"]
    if case["kind"] in ("rotate", "rotate_grad"):
        n, grad = case["n"], case["kind"] == "rotate_grad"
        table = 4 * case["rot"] * min(n, 4096)
        return {"bytes": (3 if grad else 2) * n * (hq + hk) * D * e + 4 * n + table + 2 * D * e + (8 * D if grad else 0),
                "flops": (18 if grad else 8) * n * (hq + hk) * D}
    size, prefix, length, new = (a.astype(np.int64) for a in _plan(case, 0))
    n = int(new.sum())
    if case["kind"] == "append":
        return {"bytes": 2 * n * (hq + 2 * hk) * D * e + 4 * case["rot"] * min(n, case["prefix"] + case["own"]) + 12 * len(length),
                "flops": 8 * n * (hq + hk) * D}
    shared = int(prefix.sum()) if case["groups"] else 0
    prompt = np.repeat(prefix, size)
    seen = int((new * (prompt + length - new) + new * (new + 1) // 2).sum())
    return {"bytes": 2 * (shared + int(length.sum())) * hk * D * e + 2 * n * hq * D * e, "flops": 4 * seen * hq * D}


# ---- the definitions in 64 bits ---------------------------------------------------------------------
def _rotation64(rope, position, rot, D, interleaved):
    """The rotation of each position as the partner of each element, the element's own factor and the partner's."""
    n = position.shape[0]
    cs = rope[position.long()].double()
    partner = torch.arange(D, device=rope.device)
    pair = torch.zeros(D, dtype=torch.long, device=rope.device)
    sign = torch.zeros(D, dtype=torch.float64, device=rope.device)
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        partner[a], partner[b], pair[a], pair[b], sign[a], sign[b] = b, a, i, i, -1.0, 1.0
    same = torch.ones(n, D, dtype=torch.float64, device=rope.device)
    same[:, sign != 0] = cs[:, pair[sign != 0], 0]
    cross = cs[:, pair, 1] * sign
    return partner, same, cross


def _exact_rotate(x, w, turn):
    partner, same, cross = turn
    x = x.double()
    u = x / ((x ** 2).mean(-1, keepdim=True) + EPS).sqrt() * w.double()
    return same[:, None] * u + cross[:, None] * u[..., partner]


def _exact_rotate_grad(dy, x, w, turn):
    partner, same, cross = turn
    dy, x, w = dy.double(), x.double(), w.double()
    g = same[:, None] * dy - cross[:, None] * dy[..., partner]      # the transposed rotation
    size = ((x ** 2).mean(-1, keepdim=True) + EPS).sqrt()
    gw = g * w
    dx = gw / size - x * (gw * x).sum(-1, keepdim=True) / (x.shape[-1] * size ** 3)
    return dx, (g * x / size).sum((0, 1))


def exact(case, seed):
    st = prepare(case, seed)
    kind, page, hq, hk, D = case["kind"], case.get("page"), case["hq"], case["hk"], case["D"]
    if kind in ("rotate", "rotate_grad"):
        turn = _rotation64(st["rope"], st["position"], case["rot"], D, case["interleaved"])
        if kind == "rotate":
            return {"q": _exact_rotate(st["q"], st["q_weight"], turn), "k": _exact_rotate(st["k"], st["k_weight"], turn)}
        dq, dwq = _exact_rotate_grad(st["dq"], st["q"], st["q_weight"], turn)
        dk, dwk = _exact_rotate_grad(st["dk"], st["k"], st["k_weight"], turn)
        return {"dq": dq, "dk": dk, "dq_weight": dwq, "dk_weight": dwk}
    size, prefix, length, new = _plan(case, seed)
    G = case["groups"]
    group = np.repeat(np.arange(len(size)), size)
    start = np.concatenate([[0], np.cumsum(new)])
    dev = st["q"].device
    if kind == "append":
        seq = np.repeat(np.arange(len(length)), new)
        place = np.concatenate([np.arange(int(l) - int(m), int(l)) for l, m in zip(length, new)])
        position = torch.from_numpy(prefix[group[seq]] + place).to(dev)
        turn = _rotation64(st["rope"], position, case["rot"], D, case["interleaved"])
        seq, place = torch.from_numpy(seq).to(dev), torch.from_numpy(place).to(dev)
        slot = st["pages"][seq, place // page].long()
        k, v = st["cache_k"].double(), st["cache_v"].double()
        k[slot, :, place % page] = _exact_rotate(st["k"], st["k_weight"], turn)
        v[slot, :, place % page] = st["v"].double()
        return {"q": _exact_rotate(st["q"], st["q_weight"], turn), "cache_k": k, "cache_v": v}
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=dev)

    def rows(cache, table, n):
        at = torch.arange(n, device=dev)
        return cache[table[at // page].long(), :, at % page].double()          # [n, hk, D]

    last = None
    for s in range(len(length)):
        g, m = int(group[s]), int(new[s])
        k, v = (rows(st[c], st["pages"][s], int(length[s])) for c in ("cache_k", "cache_v"))
        if G:
            if last is None or last[0] != g:
                last = (g, *(rows(st[c], st["prefix_pages"][g], int(prefix[g])) for c in ("cache_k", "cache_v")))
            k, v = torch.cat((last[1], k)), torch.cat((last[2], v))
        q = st["q"][start[s]:start[s + 1]].double().view(m, hk, hq // hk, D)
        sees = torch.arange(k.shape[0], device=dev)[None] <= torch.arange(k.shape[0] - m, k.shape[0], device=dev)[:, None]
        for h in range(hk):
            z = (q[:, h].reshape(-1, D) @ k[:, h].T).view(m, hq // hk, -1) / math.sqrt(D)
            p = torch.softmax(z.masked_fill(~sees[:, None], -math.inf), -1)
            out[start[s]:start[s + 1], h * (hq // hk):(h + 1) * (hq // hk)] = (p.view(m * (hq // hk), -1) @ v[:, h]).view(m, -1, D)
    return {"out": out}
