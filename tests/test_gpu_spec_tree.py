"""Acceptance of a token tree, greedy and drawn, against the plain walk: whole
numbers, equal in every place."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import tree
from paper_2607_01831_amd import lynx
from tests.gpu_cases import note
from tests.test_gpu_tree import random_parents

pytestmark = pytest.mark.gpu


def run(scores, tokens, parents, uniforms=None, ws=None):
    B, n = tokens.shape
    dev = [torch.as_tensor(np.ascontiguousarray(x)).cuda() for x in (scores, tokens.astype(np.int32), parents.astype(np.int32))]
    out = [torch.full(s, -7, dtype=torch.int32, device="cuda") for s in ((B,), (B, n), (B,))]
    ws = lynx.spec_tree_workspace(B, n, scores.shape[2]) if ws is None else ws
    note(f"accept_tree B={B} n={n} V={scores.shape[2]} drawn={uniforms is not None}")
    if uniforms is None:
        lynx.lynx_spec_accept_tree_greedy(*dev, *out, ws)
    else:
        lynx.lynx_spec_accept_tree_sample(*dev, torch.as_tensor(uniforms).cuda(), *out, ws)
    torch.cuda.synchronize()
    assert int(ws.max()) == 0  # left as it was found
    return [x.cpu().numpy() for x in out]


def run_way(scores, tokens, parents, uniforms, rows, looks):
    """The same by a given way of reading the rows."""
    B, n, V = *tokens.shape, scores.shape[2]
    dev = [torch.as_tensor(np.ascontiguousarray(x)).cuda() for x in (scores, tokens.astype(np.int32), parents.astype(np.int32))]
    u = None if uniforms is None else torch.as_tensor(uniforms).cuda()
    out = [torch.full(s, -7, dtype=torch.int32, device="cuda") for s in ((B,), (B, n), (B,))]
    ws = lynx.spec_tree_workspace(B, n, V)
    f = lynx.load().lynx_internal_accept_tree
    P, I = ctypes.c_void_p, ctypes.c_int32
    f.argtypes = [I, I, I, P, P, P, P, P, P, P, P, ctypes.c_size_t, I, I, P]
    note(f"accept_tree B={B} n={n} V={V} drawn={u is not None} rows={rows} looks={looks}")
    assert f(B, n, V, *[x.data_ptr() for x in dev], None if u is None else u.data_ptr(), *[x.data_ptr() for x in out],
             ws.data_ptr(), ws.nbytes, rows, looks, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert int(ws.max()) == 0
    return [x.cpu().numpy() for x in out]


def check(scores, tokens, parents, uniforms=None, ws=None):
    got, want = run(scores, tokens, parents, uniforms, ws), tree.accept_tree(scores, tokens, parents, uniforms)
    for name, g, w in zip(("accepted", "path", "next_token"), got, want):
        assert np.array_equal(g, w), (name, g, w)
    return got


def case(B, n, V, seed, drawn, agree=0.7):
    """Scores, a tree, and tokens that follow the choices with chance `agree`."""
    r = np.random.default_rng(seed)
    scores = np.round(r.standard_normal((B, n + 1, V)) * 8).astype(np.float32) / 4  # many ties
    uniforms = None
    if drawn:
        e = np.exp(scores - scores.max(-1, keepdims=True))
        scores = (e / e.sum(-1, keepdims=True)).astype(np.float32)
        uniforms = r.random((B, n + 1)).astype(np.float32)
    parents = random_parents(B, n, seed, chain=0.6)
    tokens = r.integers(0, V, (B, n))
    for b in range(B):
        for i in range(n):
            if r.random() < agree:
                row = scores[b, parents[b, i] + 1]
                tokens[b, i] = tree.choice_sample(row, uniforms[b, parents[b, i] + 1]) if drawn else tree.choice_greedy(row)
    return scores, tokens, parents, uniforms


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("B,n,V", [(1, 1, 1), (1, 1, 2), (3, 5, 7), (1, 64, 4095), (2, 63, 4096), (2, 17, 4097), (1, 8, 32000),
                                   (4, 24, 50257), (300, 3, 33), (40, 64, 100), (16, 9, 8192), (1, 2, 128256), (12, 60, 50000)])
def test_trees(B, n, V, drawn):
    check(*case(B, n, V, seed=B + n, drawn=drawn))


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("rows,looks", [(1, 0), (0, 128), (0, 1), (0, 0)])
def test_every_way_of_reading_the_rows(rows, looks, drawn):
    """All rows at once; along the path; along the path with workgroups that stop
    waiting after one look or none, so that the last one walks."""
    for i, (B, n, V) in enumerate([(1, 1, 1), (3, 5, 8193), (2, 64, 20001), (7, 33, 4096), (1, 9, 50257), (70, 6, 40)]):
        c = case(B, n, V, 20 + i, drawn, agree=0.9)
        for g, w in zip(run_way(*c, rows, looks), tree.accept_tree(*c)):
            assert np.array_equal(g, w)


@pytest.mark.parametrize("drawn", [False, True])
def test_whole_chains_and_nothing(drawn):
    s, _, _, u = case(2, 64, 500, 5, drawn)
    chain = np.tile(np.arange(64) - 1, (2, 1))
    pick = (lambda b, i: tree.choice_sample(s[b, i], u[b, i])) if drawn else (lambda b, i: tree.choice_greedy(s[b, i]))
    tokens = np.array([[pick(b, i) for i in range(64)] for b in range(2)])
    assert check(s, tokens, chain, u)[0].tolist() == [64, 64]
    tokens[0, 0] += 1
    assert check(s, tokens, chain, u)[0].tolist() == [0, 64]
    assert check(s, tokens, np.full((2, 64), -2), u)[0].tolist() == [0, 0]
    # every node a child of the context with the same token: the first
    assert check(s, np.full((2, 64), pick(1, 0)), np.full((2, 64), -1), u)[1][1, 0] == 0


@pytest.mark.parametrize("drawn", [False, True])
def test_malformed_trees_and_tokens(drawn):
    s, t, p, u = case(6, 12, 90, 11, drawn, agree=1.0)
    p[0, 3], p[1, 0], p[2, 5], p[3, 2], p[4, :] = -2, 0, 11, 2 ** 31 - 1, -2 ** 31
    check(s, t, p, u)
    t[5, ::2] = -1
    t[5, 1::4] = 90
    t[0, 0] = 2 ** 31 - 1
    check(s, t, p, u)


def test_scores_that_are_no_numbers():
    s, t, p, _ = case(5, 6, 5000, 2, False)
    s[0, 0, 1000:] = np.nan
    s[1, 0] = -np.inf
    s[2, 0] = np.nan
    s[3, 0, 17] = s[3, 0, 4999] = np.inf
    s[4, 0, :] = -np.inf
    s[4, 0, 4500] = np.nan
    t[:, 0], p[:, 0] = [tree.choice_greedy(x) for x in s[:, 0]], -1
    got = check(s, t, p)
    assert got[2][2] == -1 and got[0][2] == 0  # a choice of -1 is no node's token
    s[0, 0] = -0.0
    s[0, 0, 70] = 0.0  # equal to the others: the lowest index
    t[0, 0] = 0
    check(s, t, p)


def test_weights_at_the_edges():
    s, t, p, u = case(6, 4, 9000, 4, True)
    s[0, 0] = 0.0
    s[1, 0] = 0.0
    s[1, 0, 8999] = 1.0
    s[2, 0] = 2.0 ** -41          # below one unit each
    s[3, 0, 5:] = np.nan
    s[4, 0] = 1.5                 # clamped
    s[5, 0, :100] = -1.0
    for edge in (0.0, 1.0 - 2.0 ** -24, 1.0, -1.0, np.nan, 2.0):
        u[:, 0] = edge
        t[:, 0], p[:, 0] = [tree.choice_sample(x, edge) for x in s[:, 0]], -1
        check(s, t, p, u)


@pytest.mark.parametrize("drawn", [False, True])
def test_rows_off_the_path_may_hold_anything(drawn):
    s, t, p, u = case(3, 20, 6000, 8, drawn)
    a, path, nxt = tree.accept_tree(s, t, p, u)
    for b in range(3):
        off = [i for i in range(20) if i not in path[b, :a[b]].tolist()]
        s[b, [i + 1 for i in off]] = np.nan
        if drawn:
            u[b, [i + 1 for i in off]] = np.nan
    check(s, t, p, u)


def test_one_workspace_for_every_shape_in_graphs_too():
    """A workspace for the largest shape serves all, greedy and drawn, eager and
    in graphs whose replays alternate."""
    cases = [case(16, 24, 9000, 1, False), case(2, 64, 20000, 2, True), case(1, 3, 50, 3, False), case(9, 7, 12345, 4, True)]
    ws = torch.zeros(max(lynx.lynx_spec_tree_workspace_bytes(*c[1].shape, c[0].shape[2]) for c in cases), dtype=torch.uint8,
                     device="cuda")
    graphs, side = [], torch.cuda.Stream()
    for c in cases:
        check(*c, ws=ws)
        B, n = c[1].shape
        dev = [torch.as_tensor(np.ascontiguousarray(x)).cuda() for x in (c[0], c[1].astype(np.int32), c[2].astype(np.int32))]
        u = None if c[3] is None else torch.as_tensor(c[3]).cuda()
        out = [torch.empty(s, dtype=torch.int32, device="cuda") for s in ((B,), (B, n), (B,))]
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            if u is None:
                lynx.lynx_spec_accept_tree_greedy(*dev, *out, ws)
            else:
                lynx.lynx_spec_accept_tree_sample(*dev, u, *out, ws)
        graphs.append((g, out, dev, u))
    for turn in range(3):
        for c, (g, out, _, _) in zip(cases, graphs):
            for x in out:
                x.fill_(-7)
            note(f"replay {turn}")
            g.replay()
            torch.cuda.synchronize()
            for x, w in zip(out, tree.accept_tree(*c)):
                assert np.array_equal(x.cpu().numpy(), w)
            check(*c, ws=ws)
    assert int(ws.max()) == 0


@pytest.mark.parametrize("drawn", [False, True])
def test_calls_on_two_streams_at_once(drawn):
    """Along the path, each with a workspace of its own: whoever has to wait too
    long for the other's workgroups gives the same result."""
    calls = []
    for seed in (1, 2):
        c = case(24, 11, 128256, seed, drawn, agree=0.9)
        dev = [torch.as_tensor(np.ascontiguousarray(x)).cuda() for x in (c[0], c[1].astype(np.int32), c[2].astype(np.int32))]
        if drawn:
            dev.append(torch.as_tensor(c[3]).cuda())
        out = [torch.full(s, -7, dtype=torch.int32, device="cuda") for s in ((24,), (24, 11), (24,))]
        calls.append((dev, out, lynx.spec_tree_workspace(24, 11, 128256), torch.cuda.Stream(), tree.accept_tree(*c)))
    f = lynx.lynx_spec_accept_tree_sample if drawn else lynx.lynx_spec_accept_tree_greedy
    torch.cuda.synchronize()
    note(f"two streams drawn={drawn}")
    for _ in range(5):
        for dev, out, ws, stream, _ in calls:
            f(*dev, *out, ws, stream=stream)
    torch.cuda.synchronize()
    for _, out, ws, _, want in calls:
        assert int(ws.max()) == 0
        for x, w in zip(out, want):
            assert np.array_equal(x.cpu().numpy(), w)
