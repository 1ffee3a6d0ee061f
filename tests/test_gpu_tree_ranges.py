"""Verification of a token tree over caches whose ranges differ: values that one
token makes large, weights that are far below the largest, keys far from 0 or
with one token far from the others.  The context's kernels against the fp64
statement over the same codes.

Tolerance, for every output element, from the arithmetic of the wide kernel.  With p
the fp64 weights and o the fp64 output of a row:
 * a key is off by at most 2^-12 of its group's range, or of itself in a channel whose
   groups all reach from below 0 to above it, and by 2^-39 of the channel's largest
   (the subnormals of fp16), a query by 2^-39 of the row's largest product; fp32 sums
   of 128 products by 2^-21 of their terms (8 roundings on the way of any).  That is at most d in a score, and a row's output moves by at
   most d e^2d sum_i p_i |v_i - o|;
 * a weight is off by 2^-12 of itself and by 2^-33 of the largest one: the output by
   sum_i (2^-12 p_i + min(p_i, 2^-33)) |v_i - o|;
 * a value is off by 2^-12 of itself and 2^-39 of the segment's largest, weighted p;
 * the output is rounded to BF16: 2^-8 of it.
The other kernel (0) holds a token's weight times its V scale in fp16, against the
largest scale: 2^-11 of p times the token's range of values, and none that are 2^20
times apart; and a query times K scale in two fp16 parts: 2^-21 of the products with
the group's range.  It takes part where these bounds hold."""
import numpy as np
import pytest
import torch

from oracle import dequant, tree
from tests.gpu_cases import bits, build_cache, device_meta_to_oracle, random_bf16, random_kv
from tests.test_gpu_tree import random_parents, run

pytestmark = pytest.mark.gpu


def f64(t):
    return t.double().numpy()


def reference(c, q, kn, vn, parents, wide):
    """(outputs, tolerances), fp64 [B][n][Hq][128]."""
    B, n, Hq, D = q.shape
    G = Hq // c.Hkv
    meta = device_meta_to_oracle(c)
    out, tol = np.zeros((B, n, Hq, D)), np.zeros((B, n, Hq, D))
    for b in range(B):
        T = c.lens[b]
        K, V = dequant("full", c.OL, b, T, c.table.numpy(), c.pool.k_codes.cpu().numpy(), c.pool.v_codes.cpu().numpy(), meta)
        spread = 255.0 * np.asarray(meta.k_scale[b], np.float64)  # [Hkv][groups][128]
        zero = np.asarray(meta.k_zero[b], np.float64)
        around = ((zero <= 0) & (zero + spread >= 0))[:, :-(-T // 128)].all(1)  # [Hkv][128]
        range_v = 255.0 * np.asarray(meta.v_scale[b], np.float64)  # [Hkv][tokens]
        for h in range(c.Hkv):
            k, v, span = K[:, h], V[:, h], np.repeat(spread[h], 128, 0)[:T]
            top_k, top_v = np.abs(k).max(0), np.abs(v).max()
            for i, seen in enumerate(tree.ancestors(parents[b])):
                if seen is None:
                    continue
                x = f64(q[b, i, h * G:(h + 1) * G]) / np.sqrt(D)  # [G][128]
                keys, values = np.concatenate([k, f64(kn[b, seen, h])]), np.concatenate([v, f64(vn[b, seen, h])])
                s = x @ keys.T
                p = np.exp(s - s.max(1, keepdims=True))
                d = 2.0 ** -21 * (np.abs(x) @ np.abs(keys).T)
                d[:, :T] += 2.0 ** -12 * (np.abs(x) @ np.where(around[h], np.minimum(np.abs(k), span), span).T)
                if wide == 0:
                    d[:, :T] += 2.0 ** -21 * (np.abs(x) @ span.T)
                d += 2.0 ** -39 * (np.abs(x) @ top_k + 128 * (np.abs(x) * top_k).max(1))[:, None]
                floor = np.minimum(p, 2.0 ** -33) / p.sum(1, keepdims=True)
                p /= p.sum(1, keepdims=True)
                o = p @ values
                # (only tokens that have weight set the largest error that counts; the others' weights
                # stay below a millionth of it even e^2d times as large)
                heavy = p > 1e-9 * p.max(1, keepdims=True)
                worst = np.where(heavy, d, 0).max(1)
                off = (p * (worst * np.exp(2 * worst) + 2.0 ** -12)[:, None] + floor)
                for g in range(G):
                    dev = np.abs(values - o[g])
                    t = off[g] @ dev + 2.0 ** -12 * (p[g] @ np.abs(values)) + 2.0 ** -39 * top_v + 2.0 ** -8 * np.abs(o[g])
                    if wide == 0:
                        t += 2.0 ** -11 * (p[g, :T] @ range_v[h, :T])
                    out[b, i, h * G + g], tol[b, i, h * G + g] = o[g], t
    return out, tol


def check(c, q, kn, vn, wide, parents):
    want, tol = reference(c, q, kn, vn, parents, wide)
    got = run(c, q, kn, vn, parents, wide=wide).astype(np.float64)
    assert np.isfinite(got).all()
    err = np.abs(got - want)
    at = np.unravel_index(np.argmax(err - tol), err.shape)
    print(f"largest error {err.max():.2e}, of its tolerance at most {np.max(err / (tol + 1e-300)):.2f}")
    assert (err <= tol).all(), (at, got[at], want[at], tol[at], int((err > tol).sum()))


def made(lens, Hkv, change, bt=16, Hq=None, n=30):
    """A cache of N(0, 1) keys and values, queries and nodes, after change(k, v, q) of
    the fp32 inputs (k, v: [T][Hkv][128]; q: [n][Hq][128] of the sequence)."""
    Hq = Hq or 4 * Hkv
    ks, vs, qs = [], [], []
    for b, T in enumerate(lens):
        k, v = (x.float() for x in random_kv(T, Hkv, seed=40 + b, outlier_cols=0))
        q = random_bf16((n, Hq, 128), 70 + b).float()
        change(k, v, q)
        ks.append(k.bfloat16()), vs.append(v.bfloat16()), qs.append(q.bfloat16())
    c = build_cache(ks, vs, Hkv, bt=bt, with_oracle=False)
    B = len(lens)
    return c, torch.stack(qs), random_bf16((B, n, Hkv, 128), 5), random_bf16((B, n, Hkv, 128), 6)


@pytest.mark.parametrize("power,wide", [(8, 0), (12, 1), (20, 1), (27, 1), (20, 2), (27, 2)])
def test_a_token_of_large_values_and_no_weight(power, wide):
    def change(k, v, q):
        v[77] *= 2.0 ** power
        k[77] = -3.0 * torch.sign(q[0, 0])  # far below the others for queries of these signs
        q[:] = torch.abs(q) * torch.sign(q[0, 0])
    c, *x = made([1500, 333], 2, change)
    check(c, *x, wide, random_parents(2, 30, seed=4))


def tail(k, v, q, drop):
    k[:] = 0
    k[5, :, 0] = drop * np.sqrt(128) / 128
    q[:] = 0
    q[..., 0] = 128
    v[:] = torch.where(torch.arange(128) % 2 == 0, 1.0, 0.5)
    v[5] = 0


@pytest.mark.parametrize("wide", [1, 2])
@pytest.mark.parametrize("drop", [16.5, 17.5, 18.2])
def test_a_long_tail_of_small_weights(drop, wide):
    """One token e^drop times as heavy as every other, whose values are 0: an output is
    the tail's sum, and a kernel that drops weights of 2^-25 (e^-17.3) drops it."""
    c, q, kn, vn = made([16384, 9000], 8, lambda k, v, q: tail(k, v, q, drop), bt=None, Hq=24)
    kn[..., 0] = -4.0  # the nodes have no weight (e^-45), so that all rows are the first node's
    parents = np.full((2, 30), -1, np.int32)
    want, tol = reference(c, q[:, :1], kn[:, :1], vn[:, :1], parents[:, :1], wide)
    assert (tol < 0.03 * np.abs(want) + 1e-9).all()  # (the rounding of the weights 1 %, of the dominant score 1, of the output 0.4)
    err = np.abs(run(c, q, kn, vn, parents, wide=wide) - want)
    print(f"largest error {err.max():.2e}, of its tolerance at most {np.max(err / tol):.2f}")
    assert (err <= tol).all(), (err.max(), int((err > tol).sum()))


def offset(k, v, q, mean, query):
    """Two channels whose keys have a mean that the softmax does not see."""
    k[:, :, [3, 9]] += mean
    q[..., 3] += query
    q[..., 9] -= query


@pytest.mark.parametrize("wide", [0, 1, 2])
@pytest.mark.parametrize("mean,query", [(30, 10), (50, 20), (64, 32), (-100, 30), (1000, 10)])
def test_keys_far_from_zero(mean, query, wide):
    c, *x = made([1500, 333], 2, lambda k, v, q: offset(k, v, q, mean, query))
    check(c, *x, wide, random_parents(2, 30, seed=4))


def moving(k, v, q):
    """The mean changes from group to group, and some groups are one value."""
    offset(k, v, q, 0, 20)
    for g in range(-(-len(k) // 128)):
        k[128 * g:128 * g + 128, :, [3, 9]] += (0, 50, -70, 200)[g % 4]
    k[256:384] = 0
    k[640:768, :, 9] = 33.0


@pytest.mark.parametrize("wide", [0, 1, 2])
def test_keys_whose_mean_moves(wide):
    c, *x = made([1500, 900], 2, moving)
    check(c, *x, wide, random_parents(2, 30, seed=4))


def far_token(k, v, q, power, at):
    """A token 2^power times as large as the others, against every query's signs."""
    k[at] *= 2.0 ** power
    sign = torch.sign(q[0, :1])
    q[:] = torch.abs(q) * sign
    k[at] = -torch.abs(k[at]) * sign


@pytest.mark.parametrize("at", [77, 200])
@pytest.mark.parametrize("power,wide", [(9, 0), (10, 0), (9, 1), (10, 1), (20, 1), (9, 2), (10, 2), (20, 2)])
def test_a_token_far_from_the_others(power, at, wide):
    c, *x = made([1500, 333], 2, lambda k, v, q: far_token(k, v, q, power, at))
    check(c, *x, wide, random_parents(2, 30, seed=4))


def small_groups(k, v, q):
    """Groups a thousand and a million times smaller than the others, with queries that
    see no more of the larger ones than of them."""
    k[128:256, :, 64:] *= 2.0 ** -10
    k[:, :, :4] *= 2.0 ** 20
    k[256:384, :, :4] *= 2.0 ** -20
    q[..., :4] *= 2.0 ** -20


@pytest.mark.parametrize("wide", [0, 1, 2])
def test_groups_of_other_sizes(wide):
    c, *x = made([1500, 333], 2, small_groups)
    check(c, *x, wide, random_parents(2, 30, seed=4))


@pytest.mark.parametrize("wide", [0, 1, 2])
@pytest.mark.parametrize("sign", [1, -1])
def test_a_group_at_one_end_then_one_over_the_whole_range(sign, wide):
    """Keys less the number that the group before left: twice the largest key, of scales
    and zeros that are no BF16."""
    c, q, kn, vn = made([1500, 333], 2, lambda k, v, q: None)
    m, end = c.pool.meta, 8.0 * (1 - 2.0 ** -14)
    for d in (5, 77):
        m.k_scale[:, :, 0::2, d], m.k_zero[:, :, 0::2, d] = 2.0 ** -20, sign * (end - 2.0 ** -11)
        m.k_scale[:, :, 1::2, d], m.k_zero[:, :, 1::2, d] = 2 * end / 255, -end
    check(c, q, kn, vn, wide, random_parents(2, 30, seed=4))
