"""Host-side checks of the attention over the hierarchical cache, the head norms
with rotation and the block calls: bad arguments are refused before anything is
launched (no pointer below is dereferenced), by the C ABI and by the Python
binding."""
import ctypes
import math

import pytest
import torch

from paper_2607_01831_amd import lynx as E


@pytest.fixture(scope="module")
def lib():
    if not E.LIBRARY.exists():
        from paper_2607_01831_amd import build
        build.build()
    return E.load()


def _layout(**kw):
    base = dict(num_kv_heads=8, block_tokens=16, max_blocks_per_seq=4, num_blocks=64, max_tokens=64)
    base.update(kw)
    return E.Layout(**base)


HMETA = E.lynx_hmeta(*range(16, 144, 16))


def test_attn_hier_refusals(lib):
    def call(L=None, B=1, Hq=32, k=4, most=64, lens=16, table=16, full=0, planes=(16, 16), alpha=255.0, variant=2, meta=HMETA,
             q=16, n_tail=0, tail=(None, None), out=16, lse=None, ws=16, nws=1 << 30):
        return lib.lynx_attn_hier(ctypes.byref((L or _layout()).c()), B, Hq, k, most, lens, table, full, *planes, alpha,
                                  variant, ctypes.byref(meta), q, n_tail, *tail, out, lse, ws, nws, None)
    for bad in (dict(B=-1), dict(B=65536), dict(Hq=0), dict(Hq=12), dict(k=0), dict(k=65), dict(k=-3), dict(most=-1),
                dict(most=65), dict(lens=None), dict(lens=20), dict(table=None), dict(table=8), dict(full=2), dict(full=-1),
                dict(full=1), dict(variant=3), dict(variant=-1), dict(alpha=0.0), dict(alpha=-1.0), dict(alpha=math.nan),
                dict(alpha=math.inf), dict(alpha=2e30), dict(planes=(None, 16)), dict(planes=(16, None)),
                dict(planes=(16, 40)), dict(meta=E.lynx_hmeta(*([0] + list(range(32, 144, 16))))),
                dict(meta=E.lynx_hmeta(*(list(range(16, 128, 16)) + [100]))), dict(q=None), dict(q=8), dict(out=None),
                dict(out=12), dict(lse=4), dict(n_tail=3, tail=(16, 16)), dict(n_tail=65, tail=(16, 16)),
                dict(n_tail=-1, tail=(16, 16)), dict(n_tail=4), dict(n_tail=4, tail=(16, None)),
                dict(n_tail=4, tail=(None, 16)), dict(n_tail=4, tail=(16, 24)), dict(L=_layout(num_blocks=0))):
        assert call(**bad) == E.LYNX_EINVAL, bad
    for bad in (dict(L=_layout(head_dim=64)), dict(L=_layout(k_group_tokens=64))):
        assert call(**bad) == E.LYNX_ENOTSUP, bad
    need = E.lynx_attn_workspace_bytes(_layout(), 1, 32, 4, 64)
    for bad in (dict(ws=None), dict(ws=8), dict(nws=need - 1), dict(nws=0)):
        assert call(**bad) == E.LYNX_EWORKSPACE, bad
    assert call(B=0, lens=None, table=None, planes=(None, None), q=None, out=None, ws=None, nws=0) == E.LYNX_OK


def test_qk_norm_rope_refusals(lib):
    def call(n=4, Hq=8, Hkv=2, D=128, q=1 << 20, qs=1536, k=1 << 20, ks=1536, v=1 << 20, vs=1536, pos=16, rows=None, n_rows=4,
             qw=16, kw=16, eps=1e-6, freq=16, rotary=128, pairs=0, scale=1.0, qo=2 << 20, ko=3 << 20, vo=4 << 20):
        return lib.lynx_qk_norm_rope(n, Hq, Hkv, D, q, qs, k, ks, v, vs, pos, rows, n_rows, qw, kw, eps, freq, rotary, pairs,
                                     scale, qo, ko, vo, None)
    assert call(D=64) == E.LYNX_ENOTSUP
    for bad in (dict(n=-1), dict(Hq=0), dict(Hkv=0), dict(Hq=65537), dict(Hkv=-2), dict(q=None), dict(q=8), dict(k=None),
                dict(k=24), dict(v=None), dict(vo=None), dict(v=4), dict(vo=4), dict(qs=1023), dict(qs=1028), dict(qs=1016),
                dict(ks=255), dict(ks=260), dict(ks=-1536), dict(vs=0), dict(qs=(1 << 31) + 8), dict(pos=None), dict(pos=4),
                dict(rows=4), dict(n_rows=3), dict(n_rows=-1), dict(rows=16, n_rows=-1), dict(qw=8), dict(kw=8),
                dict(eps=-1e-6), dict(eps=math.nan), dict(eps=math.inf), dict(freq=None), dict(freq=8), dict(rotary=-16),
                dict(rotary=144), dict(rotary=24), dict(rotary=8), dict(pairs=2), dict(pairs=-1), dict(scale=math.nan),
                dict(scale=math.inf), dict(qo=None), dict(qo=8), dict(ko=None), dict(ko=8), dict(qo=1 << 20),
                dict(ko=(1 << 20) + 3 * 1536 * 2 + 512 * 2 - 16), dict(vo=(1 << 20) - 4 * 256 * 2 + 16), dict(qo=(1 << 20) - 16),
                dict(ko=2 << 20), dict(vo=3 << 20), dict(vo=(2 << 20) + 4 * 8 * 256 - 16)):
        assert call(**bad) == E.LYNX_EINVAL, bad
    none = dict(q=None, k=None, v=None, pos=None, qw=None, kw=None, freq=None, qo=None, ko=None, vo=None)
    assert call(n=0, **none) == E.LYNX_OK


def test_blocks_refusals(lib):
    K = 1 << 20  # (what lies where: no two arrays overlap)
    INS, OUTS, ARRAYS = tuple(K * i for i in range(1, 6)), (6 * K, 7 * K), tuple(K * i for i in range(8, 12))

    def extend(L=None, B=2, n_src=4, rows=8, ins=INS, outs=OUTS, arrays=ARRAYS):
        return lib.lynx_blocks_extend(ctypes.byref((L or _layout()).c()), B, n_src, rows, *ins, *outs, *arrays, None)

    def release(L=None, B=2, ins=INS):
        return lib.lynx_blocks_release(ctypes.byref((L or _layout()).c()), B, *ins, None)

    def but(t, i, p):
        return tuple(p if j == i else x for j, x in enumerate(t))
    for call in (extend, release):
        for bad in (dict(B=-1), dict(B=65536), dict(L=_layout(block_tokens=0)), dict(L=_layout(num_blocks=1 << 27)),
                    dict(L=_layout(max_blocks_per_seq=1 << 30)),
                    *(dict(ins=but(INS, i, p)) for i in range(5) for p in (None, K * (i + 1) + 8)),
                    # (lengths, counts, table, stack, its counter)
                    dict(ins=but(INS, 2, INS[0])), dict(ins=but(INS, 2, INS[1] - 16)), dict(ins=but(INS, 4, INS[0])),
                    dict(ins=but(INS, 4, INS[3])), dict(ins=but(INS, 2, INS[3]))):
            assert call(**bad) == E.LYNX_EINVAL, bad
        assert call(L=_layout(head_dim=64)) == E.LYNX_ENOTSUP
        assert call(B=0, ins=(None,) * 5) == E.LYNX_OK
    for bad in (dict(n_src=-1), dict(n_src=1 << 30), dict(rows=-1), dict(rows=(1 << 30) + 1), dict(outs=but(OUTS, 0, None)),
                dict(outs=but(OUTS, 1, None)), dict(outs=but(OUTS, 0, 6 * K + 8)), dict(arrays=but(ARRAYS, 0, 8)),
                dict(arrays=but(ARRAYS, 3, 8)), dict(outs=but(OUTS, 0, INS[1])), dict(outs=but(OUTS, 1, INS[0])),
                dict(outs=but(OUTS, 1, INS[1])), dict(outs=but(OUTS, 0, OUTS[1])), dict(arrays=but(ARRAYS, 1, INS[0])),
                dict(arrays=but(ARRAYS, 2, INS[0] - 16)), dict(arrays=but(ARRAYS, 3, INS[2])),
                dict(arrays=but(ARRAYS, 0, ARRAYS[1] + 16)), dict(arrays=but(ARRAYS, 1, INS[4]))):
        assert extend(**bad) == E.LYNX_EINVAL, bad


def _refused(call, good, **bad):
    for name, values in bad.items():
        for x in values:
            with pytest.raises((ValueError, E.LynxError)):
                call(**{**good, name: x})


def test_binding_refuses_short_and_mistyped_tensors(lib):
    """(host tensors suffice: the checks of size and type come first)"""
    z = torch.zeros
    ints = lambda *s: z(*s, dtype=torch.int32)  # noqa: E731
    b16 = lambda *s: z(*s, dtype=torch.bfloat16)  # noqa: E731
    L = _layout(num_kv_heads=2, block_tokens=64, max_blocks_per_seq=1, num_blocks=2)
    B, Hq, k, T = 2, 4, 3, 64
    plane, meta = z(L.plane_bytes(64), dtype=torch.uint8), E.HMeta.empty(L, B, device="cpu")

    def attn(lens, table, kp, vp, m, q, kt, vt, out):
        E.lynx_attn_hier(L, B, Hq, k, T, lens, table, False, kp, vp, 255.0, E.LYNX_HQ_INT4, m, q, kt, vt, out, None, None)
    short = E.HMeta(*(getattr(meta, f) for f in ("k_gmin", "k_gscale", "k_mu", "k_sigma", "v_gmin", "v_gscale", "v_mu")),
                    v_sigma=meta.v_sigma[:1])
    good = dict(lens=ints(B), table=ints(B, 1), kp=plane, vp=plane, m=meta, q=b16(B, k, Hq, 128), kt=b16(B, k, 2, 128),
                vt=b16(B, k, 2, 128), out=b16(B, k, Hq, 128))
    _refused(attn, good, lens=[ints(1), z(B)], table=[ints(1, 1)], kp=[plane[:-1], plane.view(torch.int8)], vp=[plane[1:]],
             m=[short], q=[b16(B, 1, Hq, 128), good["q"].float()], kt=[None, b16(B, k * 2, 128)], vt=[None, b16(B, 1, 2, 128)],
             out=[good["out"][:1]])

    def rope(q, k, v, pos, rows, qw, freq, qo, ko, vo):
        E.lynx_qk_norm_rope(q, k, v, pos, rows, qw, None, 1e-6, freq, False, 1.0, qo, ko, vo)
    row = b16(5, 8, 128)
    good = dict(q=row[:, :4], k=row[:, 4:6], v=row[:, 6:], pos=ints(5), rows=ints(5), qw=b16(128), freq=z(64),
                qo=b16(5, 4, 128), ko=b16(5, 2, 128), vo=b16(5, 2, 128))
    _refused(rope, good, q=[row.float()[:, :4], row[:4, :4], row[..., :64], row[:, :8:2]], k=[row[:3, 4:6], row[:, 4]],
             v=[None, row[:, 5:]], pos=[ints(4), z(5)], rows=[ints(4)], qw=[b16(64), z(128)], freq=[b16(64)],
             ko=[b16(4, 2, 128)], vo=[None, b16(4, 2, 128)])

    def extend(lens, counts, table, stack, state, granted, starts, pos):
        E.lynx_blocks_extend(L, B, 4, lens, counts, table, stack, state, granted, starts, None, pos)
    good = dict(lens=ints(B), counts=ints(B), table=ints(B, 1), stack=ints(2), state=ints(2), granted=ints(B),
                starts=ints(B + 1), pos=ints(8))
    _refused(extend, good, lens=[ints(1), z(B)], counts=[ints(1)], table=[ints(1, 1)], stack=[ints(1)], state=[ints(1)],
             granted=[ints(1)], starts=[ints(B)], pos=[z(8)])

    def release(lens, keep, table, stack, state):
        E.lynx_blocks_release(L, B, lens, keep, table, stack, state)
    _refused(release, {x: good[x] if x != "keep" else ints(B) for x in ("lens", "keep", "table", "stack", "state")},
             lens=[ints(1)], keep=[ints(1), z(B)], table=[ints(1, 1)], stack=[ints(1)], state=[ints(1)])
