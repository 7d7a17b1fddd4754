"""Plain definitions of what a rollout that drafts its tokens calls: pages and slots of a step, and the rules of sampling on logits.

Written from the formulas, one sequence and one token at a time; shares no code with the product."""
from __future__ import annotations

import numpy as np

SEQLENS, TREE, POOL = 8, 128, 256


def paths(parent):
    """The tokens on the way from each token of one tree to its root, itself among them, and whether a parent does not stand in front."""
    out, wrong = [], False
    for j, up in enumerate(parent):
        if up < -1 or up >= j:
            wrong, up = True, -1
        out.append({j} | (out[up] if up >= 0 else set()))
    return out, wrong


def plan(page, pages, ring, length, keep, add, state, n_tok, group_seq=(0,), prefix=(), parent=None):
    """The step of every sequence from `length` to keep + add.  Returns dict(pages, ring, length, state, cu_q, seq, position, slot, ancestors,
    error); lists of the new tokens alone."""
    n_seq, n_pages, error = len(length), len(ring), 0
    pages, ring = pages.copy(), ring.copy()
    most = pages.shape[1] * page
    first, count = state
    refused = 0
    for s in range(n_seq):
        if not (0 <= length[s] <= most and 0 <= keep[s] <= length[s] and add[s] >= 0 and keep[s] + add[s] <= most):
            refused = SEQLENS
        if parent is not None and add[s] > 64:
            refused = SEQLENS
    used = [-(-int(length[s]) // page) for s in range(n_seq)]
    will = [-(-int(keep[s] + add[s]) // page) for s in range(n_seq)]
    if not refused and sum(int(x) for x in add) > n_tok:
        refused = SEQLENS
    if not refused:
        taken, given = sum(max(0, w - u) for u, w in zip(used, will)), sum(max(0, u - w) for u, w in zip(used, will))
        if not (0 <= first < n_pages and 0 <= count <= n_pages) or taken > count or given > n_pages - count:
            refused = POOL
    grouped = list(group_seq)
    falls = any(a < 0 or b < a or b > n_seq for a, b in zip(grouped, grouped[1:]))
    if falls or any(p < 0 or p > 1 << 30 for p in prefix):
        error |= SEQLENS
    out = dict(pages=pages, ring=ring, length=[int(x) for x in length], state=[int(first), int(count)], cu_q=[0] * (n_seq + 1), seq=[], position=[],
               slot=[], ancestors=[], error=error | refused)
    if refused:
        return out
    tail = first + count
    t = 0
    for s in range(n_seq):
        for i in range(used[s], will[s]):
            pages[s, i] = ring[first % n_pages]
            first, count = first + 1, count - 1
        for i in range(will[s], used[s]):
            ring[tail % n_pages] = pages[s, i]
            tail, count = tail + 1, count + 1
        before = 0
        if not falls:
            for g in range(len(prefix)):
                if grouped[g] <= s < grouped[g + 1]:
                    before = int(prefix[g]) if 0 <= prefix[g] <= 1 << 30 else 0
        ways = None
        if parent is not None:
            ways, wrong = paths(parent[t:t + add[s]])
            out["error"] |= TREE if wrong else 0
        for j in range(add[s]):
            place = int(keep[s]) + j
            out["seq"].append(s)
            out["slot"].append(int(pages[s, place // page]) * page + place % page)
            out["position"].append(before + int(keep[s]) + (j if ways is None else len(ways[j]) - 1))
            if ways is not None:
                out["ancestors"].append(sum(1 << i for i in ways[j]))
        t += int(add[s])
        out["length"][s] = int(keep[s] + add[s])
        out["cu_q"][s + 1] = t
    out["state"] = [int(first % n_pages), int(count)]
    return out


def as_bits(ancestors):
    return np.array(ancestors, dtype=np.uint64).view(np.int64)


def sampling_row(logit, prompt, behind, repetition, presence, frequency, temperature, bias, allowed):
    """One row of logits [V]: `prompt` and `behind` are the tokens in front of the row's, bias {token: value}, allowed [V] of truth values
    or None.  Returns (out, lse, best, size): size [V] is the sum of the magnitudes of what is rounded on the way to out, for error bounds."""
    V = len(logit)
    x = np.array(logit, dtype=np.float64)
    size = np.zeros(V)
    count = np.zeros(V)
    seen = np.zeros(V, dtype=bool)
    for token in prompt:
        seen[token] = True
    for token in behind:
        seen[token] = True
        count[token] += 1
    for v in np.flatnonzero(seen):
        x[v] = x[v] / repetition if x[v] > 0 else x[v] * repetition
        size[v] += abs(x[v])
        if count[v]:
            size[v] += abs(frequency * count[v])
            x[v] -= frequency * count[v]
            size[v] += abs(x[v])
            x[v] -= presence
            size[v] += abs(x[v])
    for v, b in bias.items():
        x[v] += b
        size[v] += abs(x[v])
    if allowed is not None:
        x[~allowed] = -np.inf
        size[~allowed] = 0
    real = ~np.isnan(x) & (x > -np.inf)
    best = -1
    for v in np.flatnonzero(real):
        if best < 0 or x[v] > x[best]:
            best = int(v)
    out = x / temperature
    size = size / temperature + 2 * np.where(np.isfinite(out), np.abs(out), 0)
    if np.isnan(out).any():
        lse = np.nan
    elif best < 0:
        lse = -np.inf
    elif out[best] == np.inf:
        lse = np.inf
    else:
        lse = out[best] + np.log(np.exp(out - out[best]).sum())
    return out, lse, best, size
