"""Plain fp64 definitions of what stands in front of the head: norm and rotation of queries and keys with their gradient, appending to a
paged cache, and attention of sequences that stand behind shared prefixes.

Written from the formulas, one row, one token and one query at a time; shares no code with the product."""
from __future__ import annotations

import math

import numpy as np


def rope_frequencies(rot_dim, base, scaling="plain", factor=1.0, trained=0.0, slow=1.0, fast=32.0):
    if scaling == "base":
        base = base * factor ** (rot_dim / (rot_dim - 2))
    f = np.array([base ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)])
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        for i in range(len(f)):
            turns = trained * f[i] / (2 * math.pi)
            g = min(max((turns - slow) / (fast - slow), 0.0), 1.0)
            f[i] = g * f[i] + (1 - g) * f[i] / factor
    return f


def rope_table(n_pos, rot_dim, base, magnitude=1.0, **scaling):
    """[n_pos, rot_dim / 2, 2]"""
    f = rope_frequencies(rot_dim, base, **scaling)
    t = np.zeros((n_pos, rot_dim // 2, 2))
    for p in range(n_pos):
        t[p, :, 0] = magnitude * np.cos(p * f)
        t[p, :, 1] = magnitude * np.sin(p * f)
    return t


def pairs(rot_dim, interleaved):
    return [(2 * i, 2 * i + 1) if interleaved else (i, i + rot_dim // 2) for i in range(rot_dim // 2)]


def rotate(u, turn, interleaved):
    """One row; turn [rot_dim / 2, 2]."""
    y = u.copy()
    for i, (a, b) in enumerate(pairs(2 * len(turn), interleaved)):
        c, s = turn[i]
        y[a] = c * u[a] - s * u[b]
        y[b] = c * u[b] + s * u[a]
    return y


def rotate_back(dy, turn, interleaved):
    g = dy.copy()
    for i, (a, b) in enumerate(pairs(2 * len(turn), interleaved)):
        c, s = turn[i]
        g[a] = c * dy[a] + s * dy[b]
        g[b] = c * dy[b] - s * dy[a]
    return g


def norm_rope(x, weight, table, position, eps, interleaved):
    """x [n, h, D], weight [D] or None, table [n_pos, rot / 2, 2] or None; rows of zeros where the position lies outside the table."""
    y = np.zeros_like(x)
    for t in range(x.shape[0]):
        if table is not None and not 0 <= position[t] < len(table):
            continue
        for h in range(x.shape[1]):
            u = x[t, h]
            if weight is not None:
                u = u / math.sqrt(np.mean(u * u) + eps) * weight
            y[t, h] = u if table is None else rotate(u, table[position[t]], interleaved)
    return y


def norm_rope_grad(dy, x, weight, table, position, eps, interleaved):
    """(dx, d_weight or None)"""
    D = x.shape[2]
    dx = np.zeros_like(x)
    dw = None if weight is None else np.zeros(D)
    for t in range(x.shape[0]):
        if table is not None and not 0 <= position[t] < len(table):
            continue
        for h in range(x.shape[1]):
            g = dy[t, h] if table is None else rotate_back(dy[t, h], table[position[t]], interleaved)
            if weight is None:
                dx[t, h] = g
                continue
            size = math.sqrt(np.mean(x[t, h] ** 2) + eps)
            n = x[t, h] / size
            dw += g * n
            dx[t, h] = (g * weight - n * np.mean(g * weight * n)) / size
    return dx, dw


def append(cache_k, cache_v, pages, length, new, prefix, k, v):
    """Puts rows k, v [n, Hk, D] of the sequences' new tokens (new[s] of them each, in order) into copies of the cache
    [pages, Hk, page_size, D].  Returns the copies and the tokens' positions; prefix[s]: tokens in front of sequence s."""
    cache_k, cache_v = cache_k.copy(), cache_v.copy()
    size = cache_k.shape[2]
    position, t = [], 0
    for s in range(len(length)):
        for place in range(length[s] - new[s], length[s]):
            page = pages[s][place // size]
            cache_k[page, :, place % size] = k[t]
            cache_v[page, :, place % size] = v[t]
            position.append(prefix[s] + place)
            t += 1
    return cache_k, cache_v, np.array(position, dtype=np.int64)


def rows(cache, table, n):
    """The first n tokens of a page table: [n, Hk, D]."""
    size = cache.shape[2]
    out = np.zeros((n, cache.shape[1], cache.shape[3]))
    for i in range(n):
        out[i] = cache[table[i // size], :, i % size]
    return out


def attention(q, keys, values, scale, seen):
    """One sequence: q [m, Hq, D], keys and values [n, Hk, D]; query j sees the first seen[j] tokens.
    Returns out [m, Hq, D], lse [m, Hq] and, for error bounds, sum_i p_i |v_i| [m, Hq, D] and scale * max_i sum_d |q_d k_id| [m, Hq]."""
    m, Hq, D = q.shape
    share = Hq // keys.shape[1]
    out, mag = np.zeros((m, Hq, D)), np.zeros((m, Hq, D))
    lse, big = np.full((m, Hq), -np.inf), np.zeros((m, Hq))
    for j in range(m):
        n = seen[j]
        if n <= 0:
            continue
        for h in range(Hq):
            k, v = keys[:n, h // share], values[:n, h // share]
            z = scale * (k @ q[j, h])
            top = z.max()
            e = np.exp(z - top)
            out[j, h] = (e @ v) / e.sum()
            mag[j, h] = (e @ np.abs(v)) / e.sum()
            lse[j, h] = top + math.log(e.sum())
            big[j, h] = scale * (np.abs(k) @ np.abs(q[j, h])).max()
    return out, lse, mag, big
