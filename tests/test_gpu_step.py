"""A speculative step over a paged 4-bit hierarchical cache, as a server runs it: room
for the drafts out of the free blocks, the projections' heads normed and rotated at
the plan's positions into the plan's rows, attention over the context and the
drafts, and the blocks of what was dropped given back; on a ragged batch, captured
and replayed."""
import torch
import pytest

from paper_2607_01831_amd import lynx
from tests.gpu_cases import note, random_kv
from tests.hier_ref import INT4, attention
from tests.test_gpu_hier_attn import assert_inside
from tests.test_gpu_rope import EPS, freqs, reference

pytestmark = pytest.mark.gpu

ALPHA = 255.0


@pytest.mark.parametrize("whole", [True, False])
def test_speculative_step(whole, monkeypatch):
    """whole False: the binding's own form of the calls, as where its C++ is not built."""
    if not whole:
        monkeypatch.setattr(lynx, "_whole", lambda *args: None)
    lens, Hq, H, bt, k, per = [300, 5, 0, 129], 8, 2, 16, 6, 24
    B, n_blocks = len(lens), 96
    L = lynx.Layout(num_kv_heads=H, block_tokens=bt, max_blocks_per_seq=per, num_blocks=n_blocks, max_tokens=per * bt)
    ints = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    free = lynx.FreeBlocks.allocate(L, B)
    table, stack, state, zero = free.table, free.stack, free.state, ints([0] * B)
    stack.copy_(torch.randperm(n_blocks, generator=torch.Generator().manual_seed(1)))
    granted, starts = ints([0] * B), ints([0] * (B + 1))
    # the prompts' blocks, and their cache
    lynx.lynx_blocks_extend(L, B, 300, zero, ints(lens), table, stack, state, granted, starts)
    assert granted.tolist() == lens
    pool, hm = lynx.KVPool.allocate(L, B, codes=False), lynx.HMeta.empty(L, B)
    for b, n in enumerate(lens):
        kk, vv = random_kv(n, H, seed=b)
        lynx.lynx_hkv_encode(L, b, n, table, kk.cuda(), vv.cuda(), ALPHA, INT4, pool.k_anc, pool.v_anc, None, None, hm)
    # one step: k drafts a sequence
    g = torch.Generator().manual_seed(3)
    N = B * k
    qkv = torch.randn(N, Hq + 2 * H, 128, generator=g).bfloat16().cuda()
    w = [(1 + 0.2 * torch.randn(128, generator=g)).bfloat16().cuda() for _ in range(2)]
    f = freqs(128)
    d_lens, counts, after = ints(lens), ints([k] * B), ints([0] * B)
    positions, rows = (torch.empty(N, dtype=torch.int32, device="cuda") for _ in range(2))
    q, kt, vt, out = (torch.zeros(B, k, h, 128, dtype=torch.bfloat16, device="cuda") for h in (Hq, H, H, Hq))
    ws = lynx.workspace(L, B, Hq, k, L.max_tokens, tree=False)

    def step():
        lynx.lynx_blocks_extend(L, B, k, d_lens, counts, table, stack, state, granted, starts, None, positions, None, rows)
        lynx.lynx_qk_norm_rope(qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:], positions, rows, *w, EPS, f, False, 1.0, q, kt,
                               vt)
        lynx.lynx_attn_hier(L, B, Hq, k, L.max_tokens, d_lens, table, False, pool.k_anc, pool.v_anc, ALPHA, INT4, hm, q, kt, vt,
                            out, None, ws)
        torch.add(d_lens, granted, out=after)
        lynx.lynx_blocks_release(L, B, after, d_lens, table, stack, state)

    def check():
        torch.cuda.synchronize()
        assert granted.tolist() == [k] * B and positions.tolist() == [n + i for n in lens for i in range(k)]
        assert rows.tolist() == list(range(N)) and state.tolist() == [n_blocks - sum(-(-n // bt) for n in lens), 0]
        for x, weight, got in ((qkv[:, :Hq], w[0], q), (qkv[:, Hq:Hq + H], w[1], kt)):
            y, bound = reference(x, weight, positions, f, False, 1.0)
            assert ((got.view(N, -1, 128).double().cpu() - y).abs() <= bound).all()
        assert torch.equal(vt.view(N, H, 128), qkv[:, Hq + H:])
        ref, bound, lse, lse_bound = attention(L, lens, table.cpu(), (pool.k_anc.cpu(), pool.v_anc.cpu()),
                                               [getattr(hm, x).cpu() for x in lynx._HMETA_NAMES], False, ALPHA, INT4, q.cpu(),
                                               kt.cpu(), vt.cpu())
        assert_inside(out, lse, ref, bound, lse, lse_bound)
    note("step, eager")
    before = table.clone(), stack.clone()
    step()
    check()
    assert torch.equal(table, before[0]) and torch.equal(stack, before[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        qkv.copy_(torch.randn(qkv.shape, generator=g))
        note(f"step, replay {i}")
        graph.replay()
        check()
        eager = out.clone()
        step()
        assert torch.equal(out, eager)


def test_what_the_whole_calls_refuse():
    """Device tensors that are short, of another type or strided, by the calls in C++
    and by the binding's own form, which says what is wrong."""
    L = lynx.Layout(num_kv_heads=2, block_tokens=16, max_blocks_per_seq=2, num_blocks=4, max_tokens=32)
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    b16 = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    pool, hm = lynx.KVPool.allocate(L, 2, codes=False), lynx.HMeta.empty(L, 2)
    ws = lynx.workspace(L, 2, 4, 2, 32, tree=False)
    attn = dict(lens=ints(2), table=ints(2, 2), kp=pool.k_anc, vp=pool.v_anc, q=b16(2, 2, 4, 128), kt=b16(2, 3, 2, 128),
                vt=b16(2, 3, 2, 128), out=b16(2, 2, 4, 128), lse=torch.zeros(2, 2, 4, device="cuda"), ws=ws)
    row = b16(5, 8, 128)
    rope = dict(q=row[:, :4], k=row[:, 4:6], v=row[:, 6:], pos=ints(5), rows=ints(5), w=b16(128),
                f=torch.zeros(64, device="cuda"), qo=b16(5, 4, 128), ko=b16(5, 2, 128), vo=b16(5, 2, 128))
    plan = dict(lens=ints(2), counts=ints(2), table=ints(2, 2), stack=ints(4), state=ints(2), granted=ints(2), starts=ints(3),
                pos=ints(8))

    def f_attn(a):
        lynx.lynx_attn_hier(L, 2, 4, 2, 32, a["lens"], a["table"], False, a["kp"], a["vp"], 255.0, INT4, hm, a["q"], a["kt"],
                            a["vt"], a["out"], a["lse"], a["ws"])

    def f_rope(a):
        lynx.lynx_qk_norm_rope(a["q"], a["k"], a["v"], a["pos"], a["rows"], a["w"], a["w"], EPS, a["f"], True, 1.0, a["qo"],
                               a["ko"], a["vo"])

    def f_extend(a):
        lynx.lynx_blocks_extend(L, 2, 4, a["lens"], a["counts"], a["table"], a["stack"], a["state"], a["granted"], a["starts"],
                                None, a["pos"])

    def f_release(a):
        lynx.lynx_blocks_release(L, 2, a["lens"], a["counts"], a["table"], a["stack"], a["state"])
    for f, good, names in ((f_attn, attn, attn), (f_rope, rope, rope), (f_extend, plan, plan),
                           (f_release, plan, ("lens", "counts", "table", "stack", "state"))):
        f(good)
        for name in names:
            x = good[name]
            short = x[:, 1:] if f is f_rope and name in "qkv" else x.view(-1)[: x.numel() // 8]
            if name in ("qo", "f"):  # (of any size: rows, rotated dims)
                short = x.to(torch.float64)
            if f is f_extend and name == "pos":
                short = x.long()
            for bad in (short, x.cpu(), x.to(torch.float16) if x.dtype != torch.float16 else x.float(),
                        x.view(-1)[::2] if x.is_contiguous() else x[..., ::2]):
                if f is f_rope and name == "q" and bad is short:
                    bad = torch.cat([x, x], 1)[:, ::2]
                with pytest.raises((ValueError, lynx.LynxError)):
                    f({**good, name: bad})
    torch.cuda.synchronize()
