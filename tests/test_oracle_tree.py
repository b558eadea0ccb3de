"""Pins of the tree and log-probability oracles: the chain as a tree, hand-worked masks and walks, the
committed tokens' distribution, and gradients against differences."""
import numpy as np
import pytest

import oracle
from oracle import logprobs, tree


def test_masks_of_a_small_tree():
    #      0
    #    1   2
    #   3 4   5      (6: no ancestors)
    masks, depths = tree.tree_masks([-1, 0, 0, 1, 1, 2, -1])
    want = [[0], [0, 1], [0, 2], [0, 1, 3], [0, 1, 4], [0, 2, 5], [6]]
    assert [list(np.nonzero(r)[0]) for r in masks] == want
    assert list(depths) == [0, 1, 1, 2, 2, 2, 0]
    masks, depths = tree.tree_masks([-1, 0, 1, 9, 4], n_nodes=4)
    assert masks[4].sum() == 0 and depths[4] == 0 and list(np.nonzero(masks[3])[0]) == [3]


def test_chain_is_causal_attention():
    r = np.random.default_rng(0)
    N, H, KV, D, m = 5, 4, 2, 64, 7
    q, k, v = (r.standard_normal(s) for s in ((N, H, D), (m + N, KV, D), (m + N, KV, D)))
    masks, _ = tree.tree_masks(np.arange(N) - 1)
    got, mag = tree.tree_attention(q, k, v, m, masks)
    want = oracle.attention(q, k, v, m + np.arange(N) + 1)
    assert np.abs(got - want).max() < 1e-12 and (mag >= np.abs(got) - 1e-12).all()


def test_every_node_is_its_path():
    """A node's row is the last row of causal attention over the committed entries and its own line."""
    r = np.random.default_rng(1)
    N, H, KV, D, m = 9, 2, 1, 64, 3
    parents = np.array([-1, 0, 0, 1, 1, 3, 2, 6, 6])
    q, k, v = (r.standard_normal(s) for s in ((N, H, D), (m + N, KV, D), (m + N, KV, D)))
    masks, _ = tree.tree_masks(parents)
    got, _ = tree.tree_attention(q, k, v, m, masks)
    for i in range(N):
        at = np.concatenate([np.arange(m), m + np.nonzero(masks[i])[0]])
        want = oracle.attention(q[i:i + 1], k[at], v[at], np.array([len(at)]))
        assert np.abs(got[i] - want[0]).max() < 1e-12


def test_walk_by_hand():
    parents = [-1, 0, 0, 1, 1, 2]
    tokens = [50, 7, 8, 9, 9, 3]
    assert tree.tree_accept(parents, tokens, [7, 9, 0, 4, 5, 6]) == ([0, 1, 3], [7, 9, 4])   # the lower twin
    assert tree.tree_accept(parents, tokens, [1, 9, 0, 4, 5, 6]) == ([0], [1])
    assert tree.tree_accept(parents, tokens, [8, 9, 3, 4, 5, 6], n_nodes=5) == ([0, 2], [8, 3])
    assert tree.tree_accept(parents, tokens, [8, 9, 3, 4, 5, 6], n_nodes=0) == ([], [])


def test_committed_tokens_follow_the_target():
    """With next_ids drawn from the target at each node, the first two committed tokens are distributed as
    the target's, whatever the tree: chi-square over 16 pairs (15 degrees of freedom, 0.999 quantile 37.7)."""
    r = np.random.default_rng(2)
    p1 = np.array([0.5, 0.2, 0.2, 0.1])
    p2 = r.dirichlet(np.ones(4), 4)                    # after each first token
    parents, tokens = [-1, 0, 0, 1], [0, 2, 1, 3]      # drafts 2, 1, and 2-3
    trials, counts = 40000, np.zeros((4, 4))
    for _ in range(trials):
        nxt = [r.choice(4, p=p1), r.choice(4, p=p2[2]), r.choice(4, p=p2[1]), r.choice(4, p=p2[3])]
        _, out = tree.tree_accept(parents, tokens, nxt)
        second = out[1] if len(out) > 1 else r.choice(4, p=p2[out[0]])     # else the next step's
        counts[out[0], second] += 1
    want = trials * p1[:, None] * p2
    assert ((counts - want) ** 2 / want).sum() < 37.7


def test_rotation_matches_the_decoder():
    r = np.random.default_rng(3)
    x, pos = r.standard_normal((4, 2, 64)), np.array([0, 1, 17, 30000])
    want = oracle.rope(x, pos, 10000.0)
    assert np.abs(tree.append_rows(x, pos, 10000.0, 1e-6) - want).max() < 1e-9


@pytest.mark.parametrize("T", [1.0, 0.7])
def test_logprobs_and_gradient(T):
    r = np.random.default_rng(4)
    M, V = 5, 23
    z = r.standard_normal((M, V)) * 3
    z[1, ::2] = -np.inf
    z[2] = 0.25
    z[4] = -np.inf
    ids = np.array([3, 1, 7, -1, 2])
    logp, ent, top, top_lp, mx, S = logprobs.token_logprobs(z, ids, T, topk=4)
    assert list(top[2]) == [0, 1, 2, 3] and abs(ent[2] - np.log(V)) < 1e-12
    assert logp[3] == 0 and logp[4] == -np.inf and ent[4] == 0 and S[4] == 0 and list(top[4]) == [0, 1, 2, 3]
    for i in range(4):
        w = np.exp((z[i] - z[i].max()) / T)
        w /= w.sum()
        assert abs(ent[i] + sum(a * np.log(a) for a in w if a > 0)) < 1e-12
        assert abs(np.exp(top_lp[i, 0]) - w.max()) < 1e-12
    g, gh = r.standard_normal(M), r.standard_normal(M)
    grad = logprobs.token_logprobs_grad(z, ids, g, gh, T)

    def f(zz):
        lp, en = logprobs.token_logprobs(zz, ids, T)[:2]
        return (np.where(ids >= 0, g, 0) * np.where(np.isfinite(lp), lp, 0) + gh * en).sum()

    h = 1e-5
    for i in range(4):
        for x in range(V):
            if np.isneginf(z[i, x]):
                assert grad[i, x] == 0
                continue
            up, dn = z.copy(), z.copy()
            up[i, x] += h
            dn[i, x] -= h
            assert abs((f(up) - f(dn)) / (2 * h) - grad[i, x]) < 1e-8
    assert (grad[4] == 0).all()
