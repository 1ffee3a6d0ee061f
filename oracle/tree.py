"""Plain statements of the tree operators -- TEST INFRASTRUCTURE ONLY (see the
package's docstring): verification attention of a token tree in fp64, and the
acceptance walk in Python integers.  Written from the definitions in
include/lynx.h; shares nothing with the product."""
from __future__ import annotations

import numpy as np

from . import HEAD_DIM, Layout, Meta, dequant


def ancestors(parents) -> list:
    """Per node the list of its ancestors and itself, or None for a node that is
    not there (its parent is outside -1 .. i - 1, or not there itself)."""
    out = []
    for i, p in enumerate(int(x) for x in parents):
        if p == -1:
            out.append([i])
        elif 0 <= p < i and out[p] is not None:
            out.append(out[p] + [i])
        else:
            out.append(None)
    return out


def _f64(bits: np.ndarray) -> np.ndarray:
    return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def verify_tree(L: Layout, Hq: int, seq_lens, block_table, k_codes, v_codes, meta: Meta, q_bits, k_new_bits,
                v_new_bits, parents) -> np.ndarray:
    """fp64 [B][n][Hq][128]: node i over the whole context and its ancestors."""
    B, n = np.asarray(parents).shape
    G = Hq // L.Hkv
    out = np.zeros((B, n, Hq, HEAD_DIM))
    for b in range(B):
        T = int(seq_lens[b])
        K, V = dequant("full", L, b, T, block_table, k_codes, v_codes, meta) if T else (np.zeros((0, L.Hkv, HEAD_DIM)),) * 2
        kn, vn = _f64(k_new_bits[b]), _f64(v_new_bits[b])
        for i, seen in enumerate(ancestors(parents[b])):
            if seen is None:
                continue
            for h in range(Hq):
                q = _f64(q_bits[b, i, h])
                keys, values = np.concatenate([K[:, h // G], kn[seen, h // G]]), np.concatenate([V[:, h // G], vn[seen, h // G]])
                s = keys @ q / np.sqrt(HEAD_DIM)
                p = np.exp(s - s.max())
                out[b, i, h] = p @ values / p.sum()
    return out


def choice_greedy(row: np.ndarray) -> int:
    """The lowest index of the highest score; -1 where there are NaNs alone."""
    fine = ~np.isnan(row)
    if not fine.any():
        return -1
    return int(np.argmax(fine & (row == row[fine].max())))


def choice_sample(row: np.ndarray, u: float) -> int:
    """The draw with weights floor(p 2^40) and U = floor(u 2^32)."""
    r = np.where(np.isnan(row), np.float32(0), np.clip(row, np.float32(0), np.float32(1))).astype(np.float64)
    w = np.floor(r * 2.0 ** 40).astype(np.uint64)
    total = int(w.sum(dtype=np.uint64))
    if total == 0:
        return -1
    u = 0.0 if np.isnan(u) else float(u)
    U = min(max(int(u * 2 ** 32) if u > 0 else 0, 0), 2 ** 32 - 1)
    t = total * U >> 32
    return int(np.searchsorted(np.cumsum(w, dtype=np.uint64), np.uint64(t), side="right"))


def accept_tree(scores: np.ndarray, tokens, parents, uniforms=None):
    """(accepted [B], path [B][n], next_token [B]), int32."""
    B, n = np.asarray(tokens).shape
    accepted, path, nxt = np.zeros(B, np.int32), np.full((B, n), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        at, kept = -1, 0
        while True:
            row = scores[b, at + 1]
            c = choice_greedy(row) if uniforms is None else choice_sample(row, float(uniforms[b, at + 1]))
            below = [i for i in range(at + 1, n) if int(parents[b][i]) == at and int(tokens[b][i]) == c and c >= 0]
            if not below:
                break
            at = below[0]
            path[b, kept] = at
            kept += 1
        accepted[b], nxt[b] = kept, c
    return accepted, path, nxt
