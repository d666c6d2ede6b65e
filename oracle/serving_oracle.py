"""Plain fp64 numpy definitions of the calls around a verification (tree attention over a paged cache, chains from
probabilities, block tables and slot maps, accepted rows into the cache): test infrastructure only."""

import numpy as np


def lines(parent, nodes):
    """For every node the nodes from its root down to itself; an entry outside [0, n) makes node n a root."""
    out = []
    for n in range(nodes):
        p = int(parent[n])
        out.append((out[p] if 0 <= p < n else []) + [n])
    return out


def tree_attention(q, tree_k, tree_v, cache_k, cache_v, table, context, parents, nodes, window, sinks, scale):
    """q [B,N,H,D] and so on as float64 arrays, table [B,W], context [B], parents [B,N], nodes [B].
    Returns (out, weighted absolute values, largest sum of absolute products, number of seen keys), each with q's leading
    dimensions; rows behind a tree's nodes are NaN."""
    B, N, H, D = q.shape
    pages, size, KV, _ = cache_k.shape
    group = H // KV
    out = np.full(q.shape, np.nan)
    magnitude = np.full(q.shape, np.nan)
    products = np.zeros((B, N, H))
    seen = np.zeros((B, N, H), dtype=np.int64)
    for b in range(B):
        L = min(max(int(context[b]), 0), table.shape[1] * size)
        cached = [(j, int(table[b, j // size]), j % size) for j in range(L)]
        cached = [(j, p, s) for j, p, s in cached if 0 <= p < pages]
        for n, line in enumerate(lines(parents[b], min(max(int(nodes[b]), 0), N))):
            at = L + len(line) - 1

            def visible(j):
                return window <= 0 or j > at - window or j < sinks

            use = [(p, s) for j, p, s in cached if visible(j)]
            mine = [a for d, a in enumerate(line) if visible(L + d)]
            ip, js = [p for p, _ in use], [s for _, s in use]
            for h in range(H):
                kv = h // group
                k = np.concatenate([cache_k[ip, js, kv].reshape(-1, D), tree_k[b, mine, kv]])
                v = np.concatenate([cache_v[ip, js, kv].reshape(-1, D), tree_v[b, mine, kv]])
                s = k @ q[b, n, h] * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                out[b, n, h] = w @ v
                magnitude[b, n, h] = w @ np.abs(v)
                products[b, n, h] = (np.abs(k) @ np.abs(q[b, n, h])).max() * abs(scale)
                seen[b, n, h] = len(k)
    return out, magnitude, products, seen


def _mass(row):
    row = np.asarray(row, dtype=np.float64)
    return np.where(row > 0.0, row, 0.0)


def verify_chain(tokens, target, draft, uniforms):
    """One chain: tokens [n], target [n,V], draft [n,V] or None, uniforms [n] float64.  Returns (accept_len, bonus, zero mass
    found, bad token found, distance of the drawn point from the nearest step of the cumulative mass, relative)."""
    n, V = target.shape
    a, bad = 0, 0
    while a + 1 < n:
        x = int(tokens[a + 1])
        if not 0 <= x < V:
            bad = 1
            break
        p = _mass(target[a, x:x + 1])[0]
        q = _mass(draft[a, x:x + 1])[0] if draft is not None else 1.0
        if not uniforms[a + 1] * q < p:
            break
        a += 1
    row = _mass(target[a])
    zero = 0
    if a + 1 < n:
        rest = row.copy()
        if draft is not None:
            rest = np.maximum(rest - _mass(draft[a]), 0.0)
        elif not bad:
            rest[int(tokens[a + 1])] = 0.0
        if rest.sum() > 0.0:
            row = rest
        else:
            zero = 1
    c = np.cumsum(row)
    if not c[-1] > 0.0:
        return a, 0, 1, bad, 1.0
    point = uniforms[0] * c[-1]
    past = np.flatnonzero((c > point) & (row > 0.0))
    bonus = int(past[0]) if past.size else int(np.flatnonzero(row > 0.0)[-1])
    return a, bonus, zero, bad, float(np.min(np.abs(c - point)) / c[-1])


def extend_tables(table, context, new_len, free, free_count, size, slot_width, extra, packed):
    """Returns (table, context, free, free_count, granted, slots, offsets): new arrays; packed slots hold only the tokens placed."""
    pages = len(free)
    table, free = table.copy(), list(int(x) for x in free[:max(0, min(int(free_count), pages))])
    B, width = table.shape
    context = np.maximum(np.asarray(context, dtype=np.int64), 0)
    after = context.copy()
    granted = np.zeros(B, dtype=np.int64)
    for b in range(B):
        if new_len[b] < 0:
            free += [int(x) for x in table[b, :min(-(-int(context[b]) // size), width)]]
            after[b] = 0
    free = free[:pages]                            # the list holds no more
    top, asked, tokens, taken, placed = len(free), 0, 0, 0, 0
    rows, offsets = [], [0]
    for b in range(B):
        slots = []
        if new_len[b] >= 0:
            n = int(new_len[b]) + extra
            have, want = -(-int(context[b]) // size), -(-(int(context[b]) + n) // size)
            granted[b] = -1
            if want <= width and (packed or n <= slot_width):
                first = asked
                asked += want - have
                tokens += n
                if (want == have or asked <= top) and (not packed or n == 0 or tokens <= slot_width):
                    for i in range(want - have):
                        table[b, have + i] = free[top - 1 - first - i]
                    taken += want - have
                    granted[b] = n
                    after[b] = context[b] + n
                    slots = [(int(table[b, j // size]), j % size) for j in range(int(context[b]), int(after[b]))]
        rows.append(slots)
        placed += len(slots)
        offsets.append(placed)
    return table, after, free, top - taken, granted, rows, np.array(offsets)
