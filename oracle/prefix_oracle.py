"""Plain fp64 numpy definition of attention behind shared prefixes: test infrastructure only."""

import numpy as np

from oracle.serving_oracle import lines


def prefix_attention(q, tree_k, tree_v, cache_k, cache_v, table, context, parents, nodes, prefix_of, prefix_table, prefix_len, window, sinks,
                     scale):
    """serving_oracle.tree_attention with the positions of prefix prefix_of[b] (none outside [0, prefixes)) before a tree's own.
    Returns (out, weighted absolute values, largest sum of absolute products, number of seen keys, ln of the sum of exponentials)."""
    B, N, H, D = q.shape
    pages, size, KV, _ = cache_k.shape
    group = H // KV
    out, magnitude = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    products, seen, lse = np.zeros((B, N, H)), np.zeros((B, N, H), dtype=np.int64), np.full((B, N, H), np.nan)
    for b in range(B):
        rows = []                                  # (position, page, slot) of what is cached
        which = int(prefix_of[b])
        P = 0
        if 0 <= which < len(prefix_len):
            P = min(max(int(prefix_len[which]), 0), prefix_table.shape[1] * size)
            rows += [(j, int(prefix_table[which, j // size]), j % size) for j in range(P)]
        L = min(max(int(context[b]), 0), table.shape[1] * size)
        rows += [(P + j, int(table[b, j // size]), j % size) for j in range(L)]
        rows = [r for r in rows if 0 <= r[1] < pages]
        for n, line in enumerate(lines(parents[b], min(max(int(nodes[b]), 0), N))):
            at = P + L + len(line) - 1

            def visible(j):
                return window <= 0 or j > at - window or j < sinks

            use = [r for r in rows if visible(r[0])]
            mine = [a for d, a in enumerate(line) if visible(P + L + d)]
            ip, js = [r[1] for r in use], [r[2] for r in use]
            for h in range(H):
                kv = h // group
                k = np.concatenate([cache_k[ip, js, kv].reshape(-1, D), tree_k[b, mine, kv]])
                v = np.concatenate([cache_v[ip, js, kv].reshape(-1, D), tree_v[b, mine, kv]])
                s = k @ q[b, n, h] * scale
                m = s.max()
                w = np.exp(s - m)
                lse[b, n, h] = m + np.log(w.sum())
                w /= w.sum()
                out[b, n, h] = w @ v
                magnitude[b, n, h] = w @ np.abs(v)
                products[b, n, h] = (np.abs(k) @ np.abs(q[b, n, h])).max() * abs(scale)
                seen[b, n, h] = len(k)
    return out, magnitude, products, seen, lse
