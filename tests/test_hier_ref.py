"""The 64-bit reference of the attention over the hierarchical cache, pinned on the
CPU: its keys and values against the oracle's dequantization, its levels against the
oracle's tables, its attention against torch's own in 64 bits, and its bound against
keys and values rounded as the kernel rounds them.  Planted mistakes are caught."""
import math

import numpy as np
import pytest
import torch

import oracle
from paper_2607_01831_amd import inputs, lynx
from tests import hier_ref
from tests._util import bf16_bits, bits_to_f64

VARIANTS = {"biased": hier_ref.BIASED, "centred": hier_ref.CENTRED, "int4": hier_ref.INT4}
FORMS = [("biased", False), ("biased", True), ("centred", False), ("centred", True), ("int4", False)]
NAMES = lynx._HMETA_NAMES


def encoded(T, Hkv, bt, variant, alpha, seed, full):
    g = torch.Generator().manual_seed(seed)
    k, v = (torch.randn(T, Hkv, 128, generator=g).bfloat16() for _ in range(2))
    table, blocks = inputs.paged_block_table(torch.tensor([T]), bt, seed)
    OL = oracle.Layout(Hkv=Hkv, bt=bt, max_blocks=table.shape[1], max_tokens=T)
    L = lynx.Layout(num_kv_heads=Hkv, block_tokens=bt, max_blocks_per_seq=table.shape[1], num_blocks=blocks, max_tokens=T)
    n = oracle.plane_bytes(OL, blocks, 64)
    planes = {x: np.zeros(n, np.uint8) for x in ("k_anc", "v_anc", "k_res", "v_res")}
    hm = oracle.HMeta.empty(OL, 1)
    oracle.hencode(OL, 0, T, table.numpy(), bf16_bits(k), bf16_bits(v), alpha, planes, hm, variant)
    kv = [oracle.merge(planes[x + "_anc"], planes[x + "_res"]) if full else planes[x + "_anc"] for x in "kv"]
    return L, OL, table, kv, hm


@pytest.mark.parametrize("variant,full", FORMS)
@pytest.mark.parametrize("T,bt,alpha", [(1, 16, 255.0), (300, 48, 15.0), (290, 7, 1e-4)])
def test_keys_and_values_are_the_oracles(variant, full, T, bt, alpha):
    L, OL, table, kv, hm = encoded(T, 2, bt, variant, alpha, T, full)
    want = oracle.hdequant("full" if full else "anchor", OL, 0, T, table.numpy(), *kv, alpha, hm, variant)
    levels = hier_ref.level_table(alpha, VARIANTS[variant], full)
    meta = [torch.from_numpy(getattr(hm, f)) for f in NAMES]
    for i in range(2):
        top = (meta[4 * i].abs() + meta[4 * i + 1].abs()).max().item()
        for h in range(2):
            x, size = hier_ref.side(torch.from_numpy(kv[i]), *meta[4 * i:4 * i + 4], L, table, 0, h, T, full, levels)
            y = bits_to_f64(want[i]).reshape(T, 2, 128)[:, h]
            # the oracle's four fp32 roundings and half a BF16 step
            assert (np.abs(x.numpy() - y) <= 2.0 ** -8 * np.abs(y) + 2.0 ** -21 * top).all()
            assert (size >= x.abs()).all()


@pytest.mark.parametrize("variant,full", FORMS)
def test_attention_is_softmax_over_context_and_tail(variant, full):
    T, Hkv, G, k, n = 150, 2, 2, 3, 5
    L, _, table, kv, hm = encoded(T, Hkv, 16, variant, 255.0, 9, full)
    meta, planes = [torch.from_numpy(getattr(hm, f)) for f in NAMES], [torch.from_numpy(p) for p in kv]
    g = torch.Generator().manual_seed(4)
    q, kt, vt = (torch.randn(1, m, h, 128, generator=g).bfloat16() for m, h in ((k, Hkv * G), (n, Hkv), (n, Hkv)))
    out, bound, lse, lse_bound = hier_ref.attention(L, [T], table, planes, meta, full, 255.0, VARIANTS[variant], q, kt, vt)
    levels = hier_ref.level_table(255.0, VARIANTS[variant], full)
    for h in range(Hkv):
        K, dK = hier_ref.side(planes[0], *meta[:4], L, table, 0, h, T, full, levels)
        V, dV = hier_ref.side(planes[1], *meta[4:], L, table, 0, h, T, full, levels)
        heads = slice(G * h, G * h + G)
        mask = torch.arange(T + n) < torch.tensor([T + n - k + i + 1 for i in range(k)]).unsqueeze(1)

        def sdpa(K, V):
            K, V = torch.cat([K, kt[0, :, h].double()]), torch.cat([V, vt[0, :, h].double()])
            return torch.nn.functional.scaled_dot_product_attention(
                q[0, :, heads].double().transpose(0, 1), K.expand(G, -1, -1), V.expand(G, -1, -1), attn_mask=mask).transpose(0, 1)
        assert (sdpa(K, V) - out[0, :, heads]).abs().max() < 1e-12
        # keys and values off as far as they may be, either way: inside the bound
        for s in (1, -1):
            flip = torch.where(torch.rand(T, 128, generator=g) < 0.5, 1.0, -1.0) * s * 2.0 ** -11
            off = (sdpa(K + flip * dK, V - flip * dV) - out[0, :, heads]).abs()
            assert (off <= bound[0, :, heads]).all()
        # planted mistakes: a token short, a tail that is not causal, no sign, the page's minimum left out
        for bad in (sdpa(torch.cat([K[1:], K[:1] * 0]), V), sdpa(K.abs(), V), sdpa(K, V - meta[4][0, h, 0].double())):
            assert ((bad - out[0, :, heads]).abs() > bound[0, :, heads]).any()
        mask = torch.ones(k, T + n, dtype=torch.bool)
        assert ((sdpa(K, V) - out[0, :, heads]).abs() > bound[0, :, heads]).any()
    assert torch.isfinite(lse).all() and (lse_bound < 0.05).all()


def test_levels_are_the_oracles():
    for variant, full in FORMS:
        for alpha in (1e-4, 1.0, 255.0):
            _, level, alevel = oracle.htables(alpha, variant)[:3]
            got = hier_ref.level_table(alpha, VARIANTS[variant], full).numpy()
            if not full:
                want = alevel if variant == "centred" else level[np.arange(8) * (16 if variant == "biased" else 1)]
                assert np.allclose(got[:8], want, rtol=1e-6, atol=0) and np.allclose(got[15:7:-1], -want, rtol=1e-6, atol=0)
            elif variant == "centred":  # every code of both signs once
                for half in (got[:128], -got[128:]):
                    assert np.allclose(np.sort(half), np.sort(level), rtol=1e-6, atol=0)


def test_empty_queries():
    L = lynx.Layout(num_kv_heads=1, block_tokens=16, max_blocks_per_seq=1, num_blocks=1, max_tokens=16)
    meta = [torch.zeros(1, 1, 1, 128)] * 8
    plane = torch.zeros(L.plane_bytes(64), dtype=torch.uint8)
    out, _, lse, _ = hier_ref.attention(L, [0], torch.zeros(1, 1, dtype=torch.int32), (plane, plane), meta, False, 1.0, 2,
                                        torch.ones(1, 2, 1, 128).bfloat16(), None, None)
    assert (out == 0).all() and (lse == -math.inf).all()
