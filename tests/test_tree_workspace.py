"""Workspace of attention calls: what a chain of drafts asks for does not grow with
the trees' wide kernel, and a tree takes any workspace that a chain would."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2607_01831_amd import lynx

KB, PARTIAL = 1024, 128 * 4 + 8
CASES = [(1, 32, 8, 33, 32768), (4, 32, 8, 64, 8192), (2, 64, 8, 64, 65536), (16, 32, 8, 25, 8192), (1, 8, 8, 64, 4096),
         (1, 32, 8, 8, 32768), (3, 32, 4, 1, 1000)]


def layout(Hkv, T):
    return lynx.Layout(num_kv_heads=Hkv, block_tokens=T, max_blocks_per_seq=1, num_blocks=16, max_tokens=T)


@pytest.fixture(scope="module")
def lib():
    if not lynx.LIBRARY.exists():
        from paper_2607_01831_amd import build
        build.build()
    return lynx.load()


@pytest.mark.parametrize("B,Hq,Hkv,n,T", CASES)
def test_a_chain_asks_for_its_own_kernels_partials(lib, B, Hq, Hkv, n, T):
    """A row tile (32, or 16) for each of 512 workgroups at most, a partial per 512
    tokens at most, one per sequence besides, of 520 bytes."""
    rows = n * Hq
    tiles = max(512 * (32 if n * Hq // Hkv > 16 else 16), rows)
    most = 256 * KB + (min(tiles, rows * B * -(-T // 512)) + rows * B) * PARTIAL
    got, tree = (f(layout(Hkv, T), B, Hq, n, T) for f in (lynx.lynx_attn_workspace_bytes, lynx.lynx_attn_tree_workspace_bytes))
    assert got == most or n == 1 and got >= most
    assert tree == got if n * Hq // Hkv <= 64 else got <= tree <= 4 * got


def test_a_tree_workspace_serves_smaller_trees(lib):
    L = layout(8, 65536)
    sizes = [[lynx.lynx_attn_tree_workspace_bytes(L, B, 32, n, T) for n in (2, 8, 16, 17, 32, 33, 64)]  # (1: a decode's limit besides)
             for B in (1, 2, 5, 64) for T in (0, 100, 5000, 65536)]
    assert (np.diff(np.array(sizes)) >= 0).all()
    for bad in ((1, 30, 4, 64), (1, 32, 0, 64), (1, 32, 65, 64), (-1, 32, 4, 64), (1, 32, 4, -1)):
        assert lynx.lynx_attn_tree_workspace_bytes(L, *bad) == 0
    assert lynx.workspace(L, 2, 32, 64, 65536, device="cpu").nbytes == lynx.lynx_attn_tree_workspace_bytes(L, 2, 32, 64, 65536)
    assert lynx.workspace(L, 2, 32, 64, 65536, device="cpu", tree=False).nbytes == lynx.lynx_attn_workspace_bytes(L, 2, 32, 64, 65536)


def test_a_tree_refuses_less_than_a_chain_needs(lib):
    L, meta = layout(8, 65536), lynx.lynx_meta(16, 32, 48, 64)
    need = lynx.lynx_attn_workspace_bytes(L, 2, 64, 64, 65536)
    assert lib.lynx_attn_verify_tree(ctypes.byref(L.c()), 2, 64, 64, 65536, 16, 16, 16, 16, ctypes.byref(meta), 16, 16, 16, 16,
                                     16, 16, need - 1, None) == lynx.LYNX_EWORKSPACE


@pytest.mark.gpu
def test_a_tree_with_a_chains_workspace():
    """The other kernel's result where the wide one would be taken, and nothing past
    the workspace's end."""
    from tests.test_gpu_tree import cache, inputs_of, random_parents, run
    c = cache([131072 + 77], 2, 16)
    x = inputs_of(c, 8, 64)
    parents = random_parents(1, 64, seed=9)
    need = lynx.lynx_attn_workspace_bytes(c.L, 1, 8, 64, max(c.lens))
    assert need < lynx.lynx_attn_tree_workspace_bytes(c.L, 1, 8, 64, max(c.lens))
    held = torch.zeros(need + 4096, dtype=torch.uint8, device="cuda")
    held[need:] = 171
    got = run(c, *x, parents, ws=held[:need])
    assert np.array_equal(got, run(c, *x, parents, wide=0))
    assert (held[need:] == 171).all()
