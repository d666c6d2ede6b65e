"""What the oracles of the calls around a verification say on cases that can be worked out by hand."""

import numpy as np

from oracle import mpv_oracle
from oracle import serving_oracle as so


def test_a_chain_over_an_empty_cache_is_causal_attention():
    rng = np.random.default_rng(3)
    q, k, v = rng.normal(size=(3, 1, 4, 2, 8))
    none = np.zeros((0, 4, 2, 8))
    out, magnitude, _, seen = so.tree_attention(q, k, v, none, none, np.zeros((1, 0), int), [0], [[-1, 0, 1, 2]], [4], 0, 0, 0.5)
    for h in range(2):
        s = q[0, :, h] @ k[0, :, h].T * 0.5
        s[np.triu_indices(4, 1)] = -np.inf
        w = np.exp(s)
        w /= w.sum(axis=1, keepdims=True)
        assert np.allclose(out[0, :, h], w @ v[0, :, h], atol=1e-12)
    assert seen[0, :, 0].tolist() == [1, 2, 3, 4]
    assert (magnitude >= np.abs(out) - 1e-12).all()


def test_window_and_sinks_by_position():
    # values name their position, queries are zero: the output is the mean of the positions seen
    k = np.zeros((2, 4, 1, 2))
    v = np.arange(8.0).reshape(2, 4, 1, 1) * np.ones((1, 1, 1, 2))
    v = v[[1, 0]]                                  # page 1 holds positions 0 to 3
    tree = np.array([7.0, 8.0, 8.0]).reshape(1, 3, 1, 1) * np.ones((1, 1, 1, 2))
    out, *_ = so.tree_attention(np.zeros((1, 3, 1, 2)), np.zeros_like(tree), tree, k, v, np.array([[1, 0]]), [7], [[-1, 0, 0]], [3], 3, 2, 1.0)
    assert np.allclose(out[0, :, 0, 0], [(0 + 1 + 5 + 6 + 7) / 5, (0 + 1 + 6 + 7 + 8) / 5, (0 + 1 + 6 + 7 + 8) / 5])


def test_chains_agree_with_the_walk_of_the_verification_oracle():
    rng = np.random.default_rng(5)
    for _ in range(50):
        n, V = int(rng.integers(1, 5)), 9
        zt, zd = rng.normal(size=(2, n, V)).astype(np.float32)
        p, q = (np.exp(z.astype(np.float64)) / np.exp(z.astype(np.float64)).sum(1, keepdims=True) for z in (zt, zd))
        tokens = np.concatenate([[0], rng.integers(0, V, n - 1)]).astype(np.int32)
        u = rng.random(n)
        ref = mpv_oracle.verify_tree(mpv_oracle.SPECINFER, list(range(-1, n - 1)), tokens, zt, zd, 1.0, u)
        a, bonus, zero, bad, gap = so.verify_chain(tokens, p, q, u)
        if ref["min_margin"] < 1e-9 or gap < 1e-9:
            continue
        assert (a, bonus) == (ref["accept_len"], ref["bonus_token"]) and not zero and not bad


def test_chain_edge_cases():
    p = np.array([[0.5, 0.5, 0.0], [0.25, 0.25, 0.5]])
    assert so.verify_chain([0, 1], p, None, [0.6, 0.4])[:2] == (1, 2)          # accepted with 0.4 < 0.5; 0.6 of row 1 lies in token 2
    assert so.verify_chain([0, 1], p, None, [0.6, 0.5])[:2] == (0, 0)          # 0.5 < 0.5 does not hold; token 1 is taken away
    assert so.verify_chain([0, 7], p, None, [0.6, 0.0])[:4] == (0, 1, 0, 1)
    assert so.verify_chain([0, 2], p, p, [0.6, 0.0])[:3] == (0, 1, 1)          # p - q has no mass: p itself
    assert so.verify_chain([0], np.array([[0.0, np.nan, -1.0]]), None, [0.5])[:3] == (0, 0, 1)


def test_tables_by_hand():
    table = np.array([[5, -1, -1], [6, 7, -1], [8, -1, -1]])
    out = so.extend_tables(table, [3, 8, 1], [1, -1, 4], [1, 2, 9, 9, 9], 2, 4, 8, 1, False)
    t, ctx, free, count, granted, rows, offsets = out
    # request 1 gives 6 and 7 back; request 0 needs a page for its fifth token and gets 7, request 2 gets 6
    assert free == [1, 2, 6, 7] and count == 2
    assert t.tolist() == [[5, 7, -1], [6, 7, -1], [8, 6, -1]]
    assert ctx.tolist() == [5, 0, 6] and granted.tolist() == [2, 0, 5] and offsets.tolist() == [0, 2, 2, 7]
    assert rows[0] == [(5, 3), (7, 0)] and rows[2] == [(8, 1), (8, 2), (8, 3), (6, 0), (6, 1)]


def test_tables_refuse_in_order():
    table = np.full((4, 2), -1)
    t, ctx, free, count, granted, rows, _ = so.extend_tables(table, [0, 0, 0, 0], [4, 9, 5, 4], [3, 4], 2, 4, 99, 0, False)
    # 9 tokens never fit two pages; request 2 needs two and one is left, so request 3 waits behind it
    assert granted.tolist() == [4, -1, -1, -1] and count == 1 and t[0, 0] == 4
