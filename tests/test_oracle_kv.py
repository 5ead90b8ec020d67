"""The cache's oracle against properties of the definitions (no GPU)."""

import numpy as np

from oracle import kv_oracle as ko


def test_plan_moves_pages_between_pool_and_tables():
    rng = np.random.default_rng(0)
    page, cols, S, n_pool = 4, 6, 5, 20
    table = np.full((S, cols), -1)
    pool, used, length = rng.permutation(n_pool), 0, np.zeros(S, int)
    for step in range(40):
        add = rng.integers(-1, 6, S)
        o = ko.plan(length, add, pool, used, table, page, T=16)
        length, pool, used, table = o["len"], o["pool"], o["pool_used"], o["table"]
        held = [int(table[s, j]) for s in range(S) for j in range(-(-length[s] // page))]
        # every page is held by one sequence or free, none twice
        assert sorted(held + [int(p) for p in pool[used:]]) == list(range(n_pool)), step
        slots = o["slot"][o["slot"] >= 0]
        assert len(set(slots)) == len(slots) and {int(x) // page for x in slots} <= set(held)


def test_attention_of_equal_keys_is_the_mean():
    rng = np.random.default_rng(1)
    K, V = np.ones((3, 4, 2, 8)), rng.normal(size=(3, 4, 2, 8))
    table = np.array([[2, 0, -1]])
    Q = rng.normal(size=(2, 4, 8))
    out, lse, _, _, n = ko.attention(Q, K, V, table, [(np.zeros(2, int), np.array([6, 0]))], 0.5)
    v = np.concatenate([V[2], V[0, :2]])
    assert n.tolist() == [6, 0] and not out[1].any() and (lse[1] == -np.inf).all()
    for h in range(4):
        assert np.allclose(out[0, h], v[:, h // 2].mean(0))
        assert np.isclose(lse[0, h], 0.5 * Q[0, h].sum() + np.log(6))


def test_a_prefix_is_more_tokens_of_the_row():
    rng = np.random.default_rng(2)
    K, V = rng.normal(size=(2, 4, 8, 1, 4)).reshape(2, 4, 8, 1, 4)
    Q = rng.normal(size=(1, 1, 4))
    whole, lse, *_ = ko.attention(Q, K, V, np.array([[0, 1, 2]]), [(np.array([0]), np.array([21]))], 1.0)
    two, lse2, *_ = ko.attention(Q, K, V, np.array([[0, 1], [2, 3]]),
                                 [(np.array([1]), np.array([5])), (np.array([0]), np.array([16]))], 1.0)
    assert np.allclose(whole, two) and np.allclose(lse, lse2)
