"""Host-side checks of the tree, append and read-back entry points: bad
arguments are refused before anything is launched (no pointer below is
dereferenced), by the C ABI and by the Python binding."""
import ctypes

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


META = E.lynx_meta(16, 32, 48, 64)


def test_verify_tree_refusals(lib):
    def call(L=None, B=1, Hq=32, n=4, most=64, meta=META, ptrs=(16,) * 4, q=16, new=(16, 16, 16), out=16, ws=16,
             nws=1 << 30):
        return lib.lynx_attn_verify_tree(ctypes.byref((L or _layout()).c()), B, Hq, n, most, *ptrs, ctypes.byref(meta), q,
                                         *new, out, ws, nws, None)
    for bad in (dict(n=0), dict(n=65), dict(n=-1), dict(Hq=12), dict(Hq=0), dict(most=65), dict(most=-1), dict(B=-1),
                dict(B=65536), dict(new=(None, 16, 16)), dict(new=(16, None, 16)), dict(new=(16, 16, None)),
                dict(new=(16, 16, 20)), dict(new=(24, 16, 16)), dict(q=None), dict(out=None), dict(out=8),
                dict(ptrs=(16, 16, None, 16)), dict(meta=E.lynx_meta(16, 0, 48, 64)), dict(L=_layout(num_blocks=0))):
        assert call(**bad) == E.LYNX_EINVAL, bad
    assert call(L=_layout(head_dim=64)) == E.LYNX_ENOTSUP
    L = _layout()
    need = E.lynx_attn_workspace_bytes(L, 1, 32, 4, 64)
    for bad in (dict(ws=None), dict(ws=8), dict(nws=need // 64), dict(nws=0)):
        assert call(**bad) == E.LYNX_EWORKSPACE, bad
    assert call(B=0, ptrs=(None,) * 4, q=None, new=(None,) * 3, out=None, ws=None, nws=0) == E.LYNX_OK


def test_accept_tree_refusals(lib):
    assert E.lynx_spec_tree_workspace_bytes(2, 8, 5000) >= 2 * 9 * 16
    for bad in ((-1, 4, 100), (65536, 4, 100), (1, 0, 100), (1, 65, 100), (1, 4, 0), (1, 4, (1 << 23) + 1)):
        assert E.lynx_spec_tree_workspace_bytes(*bad) == 0
    need = E.lynx_spec_tree_workspace_bytes(2, 4, 100)

    def greedy(B=2, n=4, V=100, ptrs=(16,) * 6, ws=16, nws=need):
        return lib.lynx_spec_accept_tree_greedy(B, n, V, *ptrs, ws, nws, None)

    def sample(B=2, n=4, V=100, ptrs=(16,) * 7, ws=16, nws=need):
        return lib.lynx_spec_accept_tree_sample(B, n, V, *ptrs, ws, nws, None)
    for call, count in ((greedy, 6), (sample, 7)):
        for bad in (dict(B=-1), dict(B=65536), dict(n=0), dict(n=65), dict(V=0), dict(V=(1 << 23) + 1)):
            assert call(**bad) == E.LYNX_EINVAL, bad
        for i in range(count):
            for p in (None, 24):
                assert call(ptrs=tuple(p if j == i else 16 for j in range(count))) == E.LYNX_EINVAL, (i, p)
        for bad in (dict(ws=None), dict(ws=8), dict(nws=need - 1)):
            assert call(**bad) == E.LYNX_EWORKSPACE, bad
        assert call(B=0, ptrs=(None,) * count, ws=None, nws=0) == E.LYNX_OK


def test_append_refusals(lib):
    def call(L=None, B=1, most=4, n_src=8, lens=16, counts=16, path=None, table=16, new=(16, 16), ring=16,
             planes=(16,) * 6, meta=META):
        return lib.lynx_kv_append(ctypes.byref((L or _layout()).c()), B, most, n_src, lens, counts, path, table, *new, ring,
                                  *planes, ctypes.byref(meta), None)
    none = (None,) * 6
    for bad in (dict(B=-1), dict(B=65536), dict(most=-1), dict(most=8000001), dict(n_src=-1), dict(most=9),
                dict(most=65, n_src=99, path=16), dict(path=20), dict(lens=None), dict(counts=None), dict(table=None),
                dict(new=(None, 16)), dict(new=(16, None)), dict(new=(16, 24)), dict(ring=None), dict(ring=8),
                dict(planes=none), dict(planes=(16, None) + (16,) * 4), dict(planes=(None, None, None, 16, 16, 16)),
                dict(planes=(16,) * 5 + (None,)), dict(planes=(24,) + (16,) * 5), dict(meta=E.lynx_meta(0, 32, 48, 64))):
        assert call(**bad) == E.LYNX_EINVAL, bad
    assert call(L=_layout(k_group_tokens=64)) == E.LYNX_ENOTSUP
    for empty in (dict(B=0), dict(most=0)):
        assert call(**empty, lens=None, counts=None, table=None, new=(None, None), ring=None) == E.LYNX_OK
    begin = lambda L=None, B=1, ptrs=(16, 16, 16), meta=META, ring=16: lib.lynx_kv_append_begin(  # noqa: E731
        ctypes.byref((L or _layout()).c()), B, *ptrs, ctypes.byref(meta), ring, None)
    for bad in (dict(B=-1), dict(B=65536), dict(ring=None), dict(ring=24), dict(ptrs=(None, 16, 16)),
                dict(ptrs=(16, 16, 8)), dict(meta=E.lynx_meta(16, 32, 0, 64))):
        assert begin(**bad) == E.LYNX_EINVAL, bad
    assert begin(L=_layout(head_dim=64)) == E.LYNX_ENOTSUP
    assert begin(B=0, ptrs=(None,) * 3, ring=None) == E.LYNX_OK


def test_dequant_refusals(lib):
    def call(L=None, B=1, most=4, ptrs=(16,) * 5, meta=META, out=(16, 16)):
        return lib.lynx_kv_dequant(ctypes.byref((L or _layout()).c()), B, most, *ptrs, ctypes.byref(meta), *out, None)
    for bad in (dict(B=-1), dict(B=65536), dict(most=-1), dict(most=8000001), dict(out=(None, 16)), dict(out=(16, 4)),
                dict(meta=E.lynx_meta(16, 32, 48, 0)), *(dict(ptrs=tuple(None if j == i else 16 for j in range(5)))
                                                        for i in range(5))):
        assert call(**bad) == E.LYNX_EINVAL, bad
    assert call(L=_layout(head_dim=64)) == E.LYNX_ENOTSUP
    assert call(B=0, ptrs=(None,) * 5, out=(None, None)) == E.LYNX_OK
    assert call(most=0, ptrs=(None,) * 5, out=(None, None)) == E.LYNX_OK


def test_binding_refuses_short_and_mistyped_tensors(lib):
    """(host tensors suffice: the checks of size and type come first)"""
    L = _layout(num_kv_heads=2, block_tokens=64, max_blocks_per_seq=1, num_blocks=2)
    B, Hq, n, T, V = 2, 4, 3, 64, 50
    z = torch.zeros
    codes, nibbles = (z(L.plane_bytes(w), dtype=torch.uint8) for w in (128, 64))
    meta = E.Meta.empty(L, B, device="cpu")
    ints = lambda *s: z(*s, dtype=torch.int32)  # noqa: E731
    b16 = lambda *s: z(*s, dtype=torch.bfloat16)  # noqa: E731
    good = dict(lens=ints(B), table=ints(B, 1), k=codes, v=codes, meta=meta, q=b16(B, n, Hq, 128), kn=b16(B, n, 2, 128),
                vn=b16(B, n, 2, 128), parents=ints(B, n), out=b16(B, n, Hq, 128))
    ring = b16(B, E.OPEN_ROWS, 2, 128)

    def refused(call, good, **bad):
        for name, value in bad.items():
            for x in value if isinstance(value, list) else [value]:
                with pytest.raises(ValueError):
                    call(**{**good, name: x})

    f64 = E.Meta(*(x.double() for x in (meta.k_scale, meta.k_zero, meta.v_scale, meta.v_zero)))
    refused(lambda lens, table, k, v, meta, q, kn, vn, parents, out: E.lynx_attn_verify_tree(
        L, B, Hq, n, T, lens, table, k, v, meta, q, kn, vn, parents, out), good,
        lens=[ints(1), z(B, dtype=torch.int64)], table=ints(1, 1), k=[nibbles, codes.to(torch.int8)], v=nibbles, meta=f64,
        q=[good["q"][:, :2], good["q"].half()], kn=good["kn"][:1], vn=[good["vn"].float()],
        parents=[ints(B, n - 1), z(B, n, dtype=torch.int64)], out=good["out"].float())
    good = dict(s=z(B, n + 1, V), t=ints(B, n), p=ints(B, n), u=z(B, n + 1), a=ints(B), path=ints(B, n), nxt=ints(B))
    greedy = lambda s, t, p, u, a, path, nxt: E.lynx_spec_accept_tree_greedy(s, t, p, a, path, nxt, ints(0))  # noqa: E731
    sample = lambda s, t, p, u, a, path, nxt: E.lynx_spec_accept_tree_sample(s, t, p, u, a, path, nxt, ints(0))  # noqa: E731
    for call in (greedy, sample):
        refused(call, good, s=[z(B, V), good["s"].bfloat16()], t=[ints(B, n - 1), z(B, n, dtype=torch.int64)], p=ints(1, n),
                a=ints(1), path=ints(B, n - 1), nxt=z(B))
    refused(sample, good, u=[z(B, n), z(B, n + 1, dtype=torch.float64)])
    good = dict(lens=ints(B), counts=ints(B), path=ints(B, 2), table=ints(B, 1), kn=b16(B, n, 2, 128), vn=b16(B, n, 2, 128),
                ring=ring, kc=codes, vc=codes, ka=nibbles, va=nibbles, kr=nibbles, vr=nibbles, meta=meta)
    refused(lambda lens, counts, path, table, kn, vn, ring, kc, vc, ka, va, kr, vr, meta: E.lynx_kv_append(
        L, B, 2, lens, counts, path, table, kn, vn, ring, kc, vc, ka, va, kr, vr, meta), good,
        lens=ints(1), counts=z(B), path=ints(B, 1), table=ints(1, 1), kn=[good["kn"].half(), good["kn"][0]],
        vn=good["vn"][:, :2], ring=[ring[:, :255], ring.half()], kc=nibbles, va=nibbles[:-1], meta=f64)
    good = dict(lens=ints(B), table=ints(B, 1), kc=codes, meta=meta, ring=ring)
    refused(lambda lens, table, kc, meta, ring: E.lynx_kv_append_begin(L, B, lens, table, kc, meta, ring), good,
            lens=ints(1), kc=nibbles, meta=f64, ring=ring[:1])
    good = dict(s=ints(B), c=ints(B), table=ints(B, 1), kc=codes, vc=codes, meta=meta, k=b16(B, 4, 2, 128),
                v=b16(B, 4, 2, 128))
    refused(lambda s, c, table, kc, vc, meta, k, v: E.lynx_kv_dequant(L, B, 4, s, c, table, kc, vc, meta, k, v), good,
            s=ints(1), c=z(B), kc=nibbles, vc=nibbles, k=[b16(B, 3, 2, 128), z(B, 4, 2, 128)], v=b16(1, 4, 2, 128))


def test_binding_refuses_a_tensor_of_another_device(lib, monkeypatch):
    class Elsewhere:
        dtype, is_cuda, nbytes = torch.int32, True, 1 << 20

        def get_device(self):
            return 3

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    with pytest.raises(ValueError, match="device 3"):
        E.lynx_kv_append_begin(_layout(), 1, Elsewhere(), None, None, E.Meta.empty(_layout(), 1, device="cpu"), None)
