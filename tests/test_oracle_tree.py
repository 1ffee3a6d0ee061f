"""The plain tree statements against hand examples and the linear oracle: a
chain is lynx_attn_verify's causal mask and lynx_spec_accept_greedy's prefix;
a mistake planted in the mask or the walk shows."""
import numpy as np
import pytest

import oracle
from oracle import tree
from tests._util import bf16_bits


def test_ancestors_by_hand():
    #        0   1  2  3  4   5  6   7
    assert tree.ancestors([-1, 0, 0, 1, -1, 4, -2, 6]) == [[0], [0, 1], [0, 2], [0, 1, 3], [4], [4, 5], None, None]
    assert tree.ancestors([0, -1, 5, 1]) == [None, [1], None, [1, 3]]  # itself, a later node


def test_a_chain_is_the_linear_verification():
    rng = np.random.default_rng(3)
    Hkv, Hq, n, T = 2, 4, 5, 130
    L = oracle.Layout(Hkv=Hkv, bt=T, max_blocks=1, max_tokens=T)
    r = lambda *s: bf16_bits(rng.standard_normal(s))  # noqa: E731
    table = np.zeros((1, 1), np.int32)
    planes, meta = oracle.encode_batch(L, [T], table, [r(T, Hkv, 128)], [r(T, Hkv, 128)], 1)
    kc, vc = oracle.merge(planes["k_anc"], planes["k_res"]), oracle.merge(planes["v_anc"], planes["v_res"])
    q, kn, vn = r(1, n, Hq, 128), r(1, n, Hkv, 128), r(1, n, Hkv, 128)
    want, _ = oracle.verify(L, Hq, [T], table, kc, vc, meta, q, kn, vn)
    got = tree.verify_tree(L, Hq, [T], table, kc, vc, meta, q, kn, vn, [[-1, 0, 1, 2, 3]])
    assert np.allclose(got, want, rtol=1e-12, atol=1e-12)
    # siblings do not see each other: the mask matters
    other = tree.verify_tree(L, Hq, [T], table, kc, vc, meta, q, kn, vn, [[-1, -1, 1, 2, 3]])
    assert np.abs(other[0, 0] - want[0, 0]).max() < 1e-12 and np.abs(other[0, 1:] - want[0, 1:]).max() > 1e-3


@pytest.mark.parametrize("seed", range(4))
def test_a_chain_is_the_linear_acceptance(seed):
    rng = np.random.default_rng(seed)
    B, n, V = 6, 4, 7
    logits = rng.integers(0, 3, (B, n + 1, V)).astype(np.float32)  # ties
    drafts = rng.integers(0, 3, (B, n)).astype(np.int32)
    a, t = oracle.accept_greedy(logits, drafts)
    got = tree.accept_tree(logits, drafts, np.tile(np.arange(n) - 1, (B, 1)))
    assert np.array_equal(got[0], a) and np.array_equal(got[2], t)
    assert all(list(got[1][b]) == list(range(a[b])) + [-1] * (n - a[b]) for b in range(B))


def test_the_walk_by_hand():
    # choices: after the context 5, after node 0 2, after node 1 3, after node 3 9
    V, n = 10, 5
    s = np.zeros((1, n + 1, V), np.float32)
    for row, c in ((0, 5), (1, 2), (2, 3), (3, 0), (4, 9), (5, 1)):
        s[0, row, c] = 1
    parents = [[-1, -1, 1, 1, 0]]
    assert [x.tolist() for x in tree.accept_tree(s, [[4, 5, 1, 3, 2]], parents)] == [[2], [[1, 3, -1, -1, -1]], [9]]
    # the first of two children with the same token
    assert tree.accept_tree(s, [[5, 5, 1, 3, 2]], parents)[1].tolist() == [[0, 4, -1, -1, -1]]
    # a node that is not there is not walked to
    assert tree.accept_tree(s, [[4, 5, 1, 3, 2]], [[-1, -2, 1, 1, 0]])[0].tolist() == [0]


def test_draws():
    p = np.array([0.0, 0.25, 0.5, 0.25], np.float32)
    assert [tree.choice_sample(p, u) for u in (0.0, 0.2499, 0.25, 0.7499, 0.75, 0.99999)] == [1, 1, 2, 2, 3, 3]
    assert tree.choice_sample(np.zeros(3, np.float32), 0.5) == -1
    assert tree.choice_sample(np.array([np.nan, 0.1, -3], np.float32), 0.9) == 1
    assert tree.choice_greedy(np.array([np.nan, -np.inf, -np.inf], np.float32)) == 1
    assert tree.choice_greedy(np.array([np.nan], np.float32)) == -1
