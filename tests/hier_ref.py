"""Attention over the hierarchical codec's cache in 64 bits, from the planes and
metadata as they stand, and how far the kernel may be off.

The reference follows lynx.h's definition of the codec, one head at a time; it
shares nothing with the kernel.  test_gpu_hier_attn.py holds its keys and values
against lynx_hkv_dequant's, which is bit-exact against the oracle.
"""
import math

import torch

D, PAGE, CHUNK = 128, 256, 32
BIASED, CENTRED, INT4 = 0, 1, 2


def level_table(alpha, variant, full):
    """[256] or [16] signed levels, float64."""
    out = []
    for n in range(256 if full else 16):
        a, r = (n >> 4, n & 15) if full else (n, 0)
        r = r - 16 if r >= 8 else r
        V = 15 - a if a >= 8 else a
        if variant == BIASED:
            code = min(max(16 * V - r, 0), 127) if full else 16 * V
        elif variant == CENTRED:
            code = 16 * V + 8 + r if full else 16 * V + 7.5
        else:
            code = V
        lv = math.expm1(code / (7 if variant == INT4 else 127) * math.log1p(alpha)) / alpha
        out.append(-lv if a >= 8 else lv)
    return torch.tensor(out, dtype=torch.float64)


def side(plane, gmin, gscale, mu, sigma, L, table, b, h, T, full, levels):
    """(x, 2 |level b| + |m| + |x|) [T][128] of one head's keys or values; the
    tensors are on the host."""
    row = D if full else D // 2
    t = torch.arange(T)
    block = table[b].long()[t // L.block_tokens]
    raw = plane.view(-1, row)[(block * L.num_kv_heads + h) * L.block_tokens + t % L.block_tokens].long()
    if not full:
        raw = torch.stack([raw & 15, raw >> 4], -1).view(T, D)
    p = lambda x, n: x[b, h].double()[t // n]  # noqa: E731
    lb = levels[raw] * p(sigma, CHUNK) * p(gscale, PAGE)
    m = p(mu, CHUNK) * p(gscale, PAGE) + p(gmin, PAGE)
    return lb + m, 2 * lb.abs() + m.abs() + (lb + m).abs()


def attention(L, lens, table, planes, hm, full, alpha, variant, q, k_tail, v_tail):
    """(out, bound, lse, lse bound), float64 [B][k][Hq][128] and [B][k][Hq].

    The bound: every key and value is off by at most 2^-11 of side()'s second
    value, so a score by ds = sum |q| dk / sqrt(128), to which fp32 sums of 128
    products in any order add 2^-16 of sum |q k| / sqrt(128) at most; a weight by
    expm1(ds) and its own rounding, 2^-11; the output's numerator and its sum by
    those, the values' own errors and fp32 sums (2^-16); then 2^-8 of it, BF16."""
    B, k, Hq, _ = q.shape
    H, n = L.num_kv_heads, 0 if k_tail is None else k_tail.shape[1]
    levels = level_table(alpha, variant, full)
    out, bound = torch.zeros(B, k, Hq, D, dtype=torch.float64), torch.zeros(B, k, Hq, D, dtype=torch.float64)
    lse, lse_bound = torch.full((B, k, Hq), -math.inf, dtype=torch.float64), torch.zeros(B, k, Hq, dtype=torch.float64)
    for b in range(B):
        T = lens[b]
        for h in range(H):
            K, dK = side(planes[0], *hm[:4], L, table, b, h, T, full, levels)
            V, dV = side(planes[1], *hm[4:], L, table, b, h, T, full, levels)
            dK, dV = dK * 2.0 ** -11, dV * 2.0 ** -11
            if n:
                K, V = torch.cat([K, k_tail[b, :, h].double()]), torch.cat([V, v_tail[b, :, h].double()])
                dK, dV = (torch.cat([x, torch.zeros(n, D, dtype=torch.float64)]) for x in (dK, dV))
            heads = slice(h * (Hq // H), (h + 1) * (Hq // H))
            for i in range(k):
                end = T + (n - k + i + 1 if n else 0)
                if end == 0:
                    continue
                x = q[b, i, heads].double()
                s = x @ K[:end].t() / math.sqrt(D)
                ds = (x.abs() @ (dK[:end] + 2.0 ** -16 * K[:end].abs()).t()) / math.sqrt(D)
                w = torch.softmax(s, 1)
                e = torch.expm1(ds) + 2.0 ** -11 + 2.0 ** -16
                o = w @ V[:end]
                off = (w * e) @ V[:end].abs() + o.abs() * (w * e).sum(1, keepdim=True) + w @ dV[:end]
                out[b, i, heads] = o
                bound[b, i, heads] = 1.05 * off + 2.0 ** -8 * (o.abs() + off) + 1e-38
                lse[b, i, heads] = torch.logsumexp(s, 1)
                lse_bound[b, i, heads] = 1.05 * (w * e).sum(1) + 2.0 ** -20 * (1 + lse[b, i, heads].abs())
    return out, bound, lse, lse_bound
