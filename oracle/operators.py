"""Operators on a paged cache in float64 numpy, from their definitions: attention for a tree of drafted nodes, the commit of
the accepted path, accumulated attention weights, eviction by them, page means, attention over selected pages.

Arrays are those of the library's calls: pools [pages, 64, kv_heads, head_dim] of one layer (commit and eviction: [layers,
...]), page_table [batch, pages_per_row], drafted nodes [batch, nodes, ...].  Everything goes row by row and node by node.
"""
from __future__ import annotations

import numpy as np

PAGE = 64


def line_of(parents, t):
    """Node t's line in its tree: the node, its parent, and so on; a parent that does not lie before its node counts as -1."""
    line = []
    while t >= 0:
        line.append(t)
        p = int(parents[t])
        t = p if 0 <= p < t else -1
    return line


def cached(pool, table, positions):
    """Rows of the pool at these positions of a sequence."""
    positions = np.asarray(positions, np.int64)
    return pool[table[positions // PAGE], positions % PAGE].astype(np.float64)


def positions_of(table, n_pages, positions):
    """Those of the positions whose page lies in the pool."""
    return [s for s in positions if 0 <= table[s // PAGE] < n_pages]


def softmax_row(q, keys, values, scale):
    """One query: output and log of the softmax's sum (0 and -inf where it sees nothing)."""
    if len(keys) == 0:
        return np.zeros(values.shape[-1]), -np.inf
    s = keys @ q * scale
    w = np.exp(s - s.max())
    return w @ values / w.sum(), s.max() + np.log(w.sum())


def attention(q, k_new, v_new, k_pool, v_pool, table, lens, parents, nodes, scale, seen=None):
    """out [batch, nodes, heads, head_dim], lse.  seen(b, t, h): the cached positions that node t sees under key head h (all below
    the length if not given)."""
    b_all, t_all, heads, d = q.shape
    hk = k_new.shape[2]
    out, lse = np.zeros((b_all, t_all, heads, v_new.shape[-1])), np.full((b_all, t_all, heads), -np.inf)
    for b in range(b_all):
        for t in range(nodes[b]):
            line = line_of(parents[b], t)
            for h in range(hk):
                at = positions_of(table[b], len(k_pool), range(lens[b]) if seen is None else seen(b, t, h))
                keys = np.concatenate([cached(k_pool[:, :, h], table[b], at).reshape(-1, d), k_new[b, line, h].astype(np.float64)])
                values = np.concatenate([cached(v_pool[:, :, h], table[b], at).reshape(-1, d), v_new[b, line, h].astype(np.float64)])
                for g in range(h * heads // hk, (h + 1) * heads // hk):
                    out[b, t, g], lse[b, t, g] = softmax_row(q[b, t, g].astype(np.float64), keys, values, scale)
    return out, lse


def page_means(k_pool, table, lens):
    """[batch, pages_per_row, kv_heads, head_dim]: means of the full pages, as they are held in 32 bits; NaN elsewhere."""
    means = np.full(table.shape + k_pool.shape[2:], np.nan, np.float32)
    for b, n in enumerate(lens):
        for p in range(n // PAGE):
            means[b, p] = k_pool[table[b, p]].astype(np.float64).sum(0) / PAGE
    return means


def select_pages(q, means, lens, nodes, select):
    """int32 [batch, nodes, kv_heads, select], ascending, -1 behind the last."""
    b_all, t_all, heads, _ = q.shape
    hk = means.shape[2]
    pages = np.full((b_all, t_all, hk, select), -1, np.int32)
    for b in range(b_all):
        full = lens[b] // PAGE
        for t in range(nodes[b]):
            for h in range(hk):
                score = means[b, :full, h].astype(np.float64) @ q[b, t, h * heads // hk:(h + 1) * heads // hk].astype(np.float64).sum(0)
                best = sorted(range(full), key=lambda p: (np.isnan(score[p]), -score[p] if score[p] == score[p] else 0.0, p))[:select]
                pages[b, t, h, :len(best)] = sorted(best)
    return pages


def page_attention(q, k_new, v_new, k_pool, v_pool, table, means, lens, parents, select, nodes, scale):
    pages = select_pages(q, means, lens, nodes, select)

    def seen(b, t, h):
        chosen = [p * PAGE + s for p in pages[b, t, h] if p >= 0 for s in range(PAGE)]
        return chosen + list(range(lens[b] // PAGE * PAGE, lens[b]))
    return attention(q, k_new, v_new, k_pool, v_pool, table, lens, parents, nodes, scale, seen) + (pages,)


def accept_path(parents, tokens, top1, last_top1, nodes, room, eos_id=-1):
    """One row's walk: the nodes taken, and the prediction after the last of them."""
    path, at, want = [], -1, last_top1
    while len(path) < room:
        child = [u for u in range(nodes) if u > at and (parents[u] if 0 <= parents[u] < u else -1) == at and tokens[u] == want]
        if not child:
            break
        at = child[0]
        path.append(at)
        want = top1[at]
        if eos_id >= 0 and tokens[at] == eos_id:
            break
    return path, want


def commit(k_new, v_new, k_pool, v_pool, table, lens, parents, tokens, top1, last_top1, nodes, eos_id=-1):
    """New lengths, accepted counts, paths, next predictions and the pools [layers, ...] after the commit."""
    k_pool, v_pool = k_pool.copy(), v_pool.copy()
    b_all, t_all = parents.shape
    paths, accepted, following = np.full((b_all, t_all), -1, np.int32), np.zeros(b_all, np.int32), np.zeros(b_all, np.int32)
    for b in range(b_all):
        room = table.shape[1] * PAGE - lens[b]
        path, following[b] = accept_path(parents[b], tokens[b], top1[b], last_top1[b], nodes[b], room, eos_id)
        accepted[b] = len(path)
        paths[b, :len(path)] = path
        for i, u in enumerate(path):
            page = table[b, (lens[b] + i) // PAGE]
            if 0 <= page < k_pool.shape[1]:
                k_pool[:, page, (lens[b] + i) % PAGE], v_pool[:, page, (lens[b] + i) % PAGE] = k_new[:, b, u], v_new[:, b, u]
    return np.asarray(lens) + accepted, accepted, paths, following, k_pool, v_pool


def cache_weights(q, lse, path, accepted, k_pool, table, lens, seen, weights, positions, scale):
    """weights (float64) and positions [batch, kv_heads, capacity] after the step."""
    weights, positions = weights.astype(np.float64), positions.copy()
    heads, hk = q.shape[2], weights.shape[1]
    for b in range(len(lens)):
        n, got = lens[b], accepted[b]
        if got:
            weights[b, :, n:n + got] = 0.0
            positions[b, :, n:n + got] = seen[b] + np.arange(got)
        for i in range(got):
            at = positions_of(table[b], len(k_pool), range(n + i + 1))
            for g in range(heads):
                h = g * hk // heads
                s = cached(k_pool[:, :, h], table[b], at) @ q[b, path[b, i], g].astype(np.float64) * scale
                weights[b, h, at] += np.exp(s - np.float64(lse[b, path[b, i], g]))
    return weights, positions


def evict(weights, positions, k_pool, v_pool, table, lens, seen, budget, recent):
    """New lengths, weights, positions and pools [layers, ...] after an eviction."""
    weights, positions, k_pool, v_pool = weights.copy(), positions.copy(), k_pool.copy(), v_pool.copy()
    layers, b_all, hk, _ = weights.shape
    for b in range(b_all):
        if lens[b] <= budget:
            continue
        for layer in range(layers):
            for h in range(hk):
                w, p = weights[layer, b, h], positions[layer, b, h]

                def rank(s):
                    return (p[s] < seen[b] - recent, np.isnan(w[s]), -w[s] if w[s] == w[s] else 0.0, s)
                kept = sorted(sorted(range(lens[b]), key=rank)[:budget])
                stays = set(kept)
                holes = [s for s in range(budget) if s not in stays]
                for to, source in zip(holes, [s for s in kept if s >= budget]):
                    w[to], p[to] = w[source], p[source]
                    for pool in (k_pool, v_pool):
                        pool[layer, table[b, to // PAGE], to % PAGE, h] = pool[layer, table[b, source // PAGE], source % PAGE, h]
    return np.minimum(lens, budget), weights, positions, k_pool, v_pool
