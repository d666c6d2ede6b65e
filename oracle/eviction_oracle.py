"""Plain fp64 numpy definitions of the weight that cached positions gather and of their eviction: test infrastructure only."""

import numpy as np


def score_positions(q, tree_k, cache_k, table, context, lse, scores, accept, path_nodes, scale, decay):
    """q [layers,B,N,H,D], tree_k [layers,B,N,KV,D], cache_k [layers,pages,size,KV,D], lse [layers,B,N,H], scores [layers,B,G,width] as
    float64; accept [B], path_nodes [B][..].  Returns (scores, bound): the new scores, and what a relative error e of a weight's exponent
    (times the exponent's terms' sizes) makes of them, per unit of e."""
    layers, B, N, H, D = q.shape
    pages, size, KV = cache_k.shape[1:4]
    G, width = scores.shape[2:]
    group = H // KV
    scores = scores.copy()
    bound = np.zeros_like(scores)
    for b in range(B):
        L = min(max(int(context[b]), 0), table.shape[1] * size)
        nodes = [0] + [int(x) for x in path_nodes[b][:accept[b]]]
        keys = []                                  # (position, where its key is)
        for j in range(L):
            page = int(table[b, j // size])
            if 0 <= page < pages:
                keys.append((j, ("cache", page, j % size)))
        keys += [(L + i, ("tree", n)) for i, n in enumerate(nodes) if 0 <= n < N]
        keys = [k for k in keys if k[0] < width]
        bound[:, b, :, :min(L, width)] += np.abs(decay * scores[:, b, :, :min(L, width)])
        scores[:, b, :, :min(L, width)] *= decay
        scores[:, b, :, L:L + len(nodes)] = 0.0
        for layer in range(layers):
            for j, where in keys:
                k = cache_k[layer, where[1], where[2]] if where[0] == "cache" else tree_k[layer, b, where[1]]
                for i, n in enumerate(nodes):
                    if not 0 <= n < N or j > L + i:
                        continue
                    for h in range(H):
                        s = scale * (q[layer, b, n, h] @ k[h // group])
                        big = abs(scale) * (np.abs(q[layer, b, n, h]) @ np.abs(k[h // group]))
                        if lse[layer, b, n, h] == -np.inf:
                            continue
                        w = np.exp(s - lse[layer, b, n, h])
                        g = h // group if G > 1 else 0
                        scores[layer, b, g, j] += w
                        if w > 0.0:
                            bound[layer, b, g, j] += w * (big + abs(lse[layer, b, n, h]) + abs(s))
    return scores, bound


def evict_positions(cache_k, cache_v, table, context, scores, free, free_count, budget, trigger, sinks, recent):
    """cache_k / cache_v [layers,pages,size,KV,D], scores [layers,B,G,width].  Returns (cache_k, cache_v, scores, kept, free list, context):
    new arrays; scores behind a request's positions are NaN."""
    cache_k, cache_v = cache_k.copy(), cache_v.copy()
    layers, pages, size, KV = cache_k.shape[:4]
    B, G, width = scores.shape[1:]
    new = np.full(scores.shape, np.nan)
    kept = np.full((layers, B, G, budget), -1, dtype=np.int64)
    free = [int(x) for x in free[:min(max(int(free_count), 0), pages)]]
    after = []
    for b in range(B):
        L = min(max(int(context[b]), 0), table.shape[1] * size)
        after.append(min(L, budget) if L > trigger else L)
        if L <= trigger:
            new[:, b, :, :L] = scores[:, b, :, :L]
            continue
        free += [int(x) for x in table[b, -(-budget // size):-(-L // size)] if 0 <= x < pages]
        for layer in range(layers):
            for g in range(G):
                row = scores[layer, b, g]
                middle = sorted(range(sinks, L - recent), key=lambda j: (-np.inf if np.isnan(row[j]) else row[j], -j), reverse=True)
                # (reverse of ascending (score, -index): larger scores first, of equal ones the lower index)
                keep = sorted(list(range(sinks)) + middle[:budget - sinks - recent] + list(range(L - recent, L)))
                kept[layer, b, g] = keep
                new[layer, b, g, :budget] = row[keep]
                heads = slice(g, g + 1) if G > 1 else slice(None)
                for i, j in enumerate(keep):
                    to, where = int(table[b, i // size]), int(table[b, j // size])
                    if 0 <= to < pages and 0 <= where < pages:
                        cache_k[layer, to, i % size, heads] = cache_k[layer, where, j % size, heads]
                        cache_v[layer, to, i % size, heads] = cache_v[layer, where, j % size, heads]
    return cache_k, cache_v, new, kept, free[:pages], after
