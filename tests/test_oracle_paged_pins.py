"""Pins of the oracle's paged and tree functions: causal queries are the multi-query oracle, a tree's node is a decode query over
its own path laid out as a plain sequence, and a plan's books balance over a server's life."""
import numpy as np
import pytest

from oracle import elitekv_oracle as orc


def _draw(seed, S, n_h=3, d_h=16, r=2, d_c=12, d_ck=0):
    rng = np.random.default_rng(seed)
    dk, dv = (d_ck, d_c - d_ck) if d_ck else (d_c, d_c)
    idx = np.stack([rng.choice(d_h // 2, r, replace=False) for _ in range(n_h)])
    return rng, idx, rng.standard_normal((S, n_h, 2 * r)), rng.standard_normal((S, d_c)), rng.standard_normal(
        (dk, n_h, d_h - 2 * r)), rng.standard_normal((dv, n_h, d_h))


@pytest.mark.parametrize("d_ck", [0, 5])
def test_causal_queries_are_the_multiquery_oracle(d_ck):
    S, T = 11, 4
    rng, idx, ke, c, W_uk, W_uv = _draw(1, S, d_ck=d_ck)
    q, kv = rng.standard_normal((T, 3, 16)), np.array([0, 3, 10, 11])
    pos = np.maximum(kv - 1, 0)
    got = orc.seen_attn(q, pos, ke, c, np.arange(S)[None] < kv[:, None], W_uk, W_uv, idx, 16, 100.0, d_ck)
    if d_ck:
        want = orc.slrd_multiquery_attn(q[None], pos[None], [ke], [c[:, :d_ck]], [c[:, d_ck:]], kv[None], W_uk, W_uv, idx, 16, 100.0)[0]
    else:
        want = orc.multiquery_attn(q[None], pos[None], [ke], [c], kv[None], W_uk, W_uv, idx, 16, 100.0)[0]
    np.testing.assert_allclose(got, want, rtol=0, atol=1e-14)


def test_a_node_is_a_decode_query_over_its_own_path():
    P, parent = 5, [-1, 0, 0, 1, 2, 2, -1, 6]
    T, S = len(parent), 5 + len(parent)
    rng, idx, ke, c, W_uk, W_uv = _draw(2, S)
    sees = orc.tree_sees(parent, T)
    depth = sees.sum(axis=1) - 1
    assert depth.tolist() == [0, 1, 1, 2, 2, 2, 0, 1]
    q = rng.standard_normal((T, 3, 16))
    seen = np.concatenate([np.ones((T, P), dtype=bool), sees], axis=1)
    got = orc.seen_attn(q, P + depth, ke, c, seen, W_uk, W_uv, idx, 16, 100.0)
    for t in range(T):
        path = [t]
        while parent[path[0]] >= 0:
            path.insert(0, parent[path[0]])
        rows = list(range(P)) + [P + j for j in path]
        want = orc.decode_attn(q[t][None], [P + len(path) - 1], [ke[rows]], [c[rows]], [len(rows)], W_uk, W_uv, idx, 16, 100.0)[0]
        np.testing.assert_allclose(got[t], want, rtol=0, atol=1e-14)
    # rows that nobody sees do not matter, whatever they hold
    ke[P + 7], c[P + 7] = np.nan, np.inf
    again = orc.seen_attn(q[:7], (P + depth)[:7], ke, c, seen[:7], W_uk, W_uv, idx, 16, 100.0)
    np.testing.assert_array_equal(again, got[:7])


def test_bad_parents_are_roots_and_words_hold_the_bits():
    sees = orc.tree_sees([3, 0, 9, -7], 4)
    assert sees.tolist() == [[1, 0, 0, 0], [1, 1, 0, 0], [0, 0, 1, 0], [0, 0, 0, 1]]
    wide = np.zeros((2, 70), dtype=bool)
    wide[0, [0, 31, 32, 69]] = True
    assert orc.mask_words(wide).tolist() == [[0x80000001, 1, 1 << 5], [0, 0, 0]]


def test_books_balance_over_a_servers_life():
    rng = np.random.default_rng(3)
    B, cols, page, n_pages, T = 6, 5, 16, 17, 3
    table, held, free, span = np.full((B, cols), -1), np.zeros(B, int), np.arange(n_pages), np.array([0, n_pages])
    cached = np.zeros(B, int)
    short = 0
    for _ in range(400):
        new = rng.integers(0, T + 1, B)
        gone = rng.random(B) < 0.03
        cached[gone], new[gone] = 0, 0
        table, held, free, span, pos, slot, kv = orc.page_plan(cached, new, T, page, n_pages, table, held, free, span)
        mine = [p for b in range(B) for p in table[b, :held[b]]]
        spare = [free[i % n_pages] for i in range(span[0], span[1])]
        assert sorted(mine + spare) == list(range(n_pages))
        rows = slot[slot >= 0]
        assert len(set(rows)) == len(rows) and ((kv > 0) == (slot >= 0)).all()
        stored = (slot >= 0).sum(axis=1)
        short += int((stored < new).any())
        cached = np.where(stored < new, cached, cached + stored)
    assert short > 0                                       # the pool did run dry
