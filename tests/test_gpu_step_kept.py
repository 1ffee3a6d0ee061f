"""Steps that keep some of their drafts: the plan's blocks are filled by the append or
stand behind the cache as a tail, the rest goes back, sequences end and others begin
in their place, some are refused for want of blocks; eager, and captured and replayed."""
import math

import pytest
import torch

from paper_2607_01831_amd import lynx
from tests.gpu_cases import note, random_kv
from tests.hier_ref import INT4, attention
from tests.test_gpu_hier_attn import assert_inside
from tests.test_gpu_rope import EPS, freqs, reference

pytestmark = pytest.mark.gpu

ints = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731


class Server:
    """A batch over the uniform codec's paged cache, whose steps run on the device alone."""

    def __init__(self, B, k, bt, per, n_blocks, Hq=8, H=2):
        self.B, self.k, self.Hq, self.H = B, k, Hq, H
        self.L = lynx.Layout(num_kv_heads=H, block_tokens=bt, max_blocks_per_seq=per, num_blocks=n_blocks, max_tokens=per * bt)
        self.free = lynx.FreeBlocks.allocate(self.L, B)
        self.free.stack.copy_(torch.randperm(n_blocks, generator=torch.Generator().manual_seed(1)))
        self.pool, self.ring = lynx.KVPool.allocate(self.L, B), None
        self.ring = self.pool.open_rows()
        self.lens, self.granted, self.starts = ints([0] * B), ints([0] * B), ints([0] * (B + 1))
        self.kept = ints([0] * B)                       # tokens appended by the step
        self.asked, self.accept, self.done = ints([0] * B), ints([0] * B), torch.zeros(B, dtype=torch.bool, device="cuda")
        bf = lambda h: torch.zeros(B, k, h, 128, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.q, self.kn, self.vn, self.out = bf(Hq), bf(H), bf(H), bf(Hq)
        self.qkv = torch.zeros(B * k, Hq + 2 * H, 128, dtype=torch.bfloat16, device="cuda")
        self.plan = [ints([0] * (B * k)) for _ in range(4)]  # seq_of, positions, slots, rows
        g = torch.Generator().manual_seed(2)
        self.w = [(1 + 0.2 * torch.randn(128, generator=g)).bfloat16().cuda() for _ in range(2)]
        self.f, self.ws = freqs(128), lynx.workspace(self.L, B, Hq, k, self.L.max_tokens, tree=False)
        self.before = torch.zeros_like(self.free.table)  # the table while the step's blocks stand in it
        # on the host: what every sequence is made of
        self.host = [[torch.zeros(0, H, 128, dtype=torch.bfloat16) for _ in range(2)] for _ in range(B)]

    def step(self):
        L, B, f, Hq, H = self.L, self.B, self.free, self.Hq, self.H
        lynx.lynx_blocks_extend(L, B, self.k, self.lens, self.asked, f.table, f.stack, f.state, self.granted, self.starts, *self.plan)
        lynx.lynx_qk_norm_rope(self.qkv[:, :Hq], self.qkv[:, Hq:Hq + H], self.qkv[:, Hq + H:], self.plan[1], self.plan[3], *self.w,
                               EPS, self.f, False, 1.0, self.q, self.kn, self.vn)
        lynx.lynx_attn_verify(L, B, Hq, self.k, L.max_tokens, self.lens, f.table, self.pool.k_codes, self.pool.v_codes,
                              self.pool.meta, self.q, self.kn, self.vn, self.out, self.ws)
        torch.minimum(self.accept, self.granted, out=self.kept)
        self.pool.append(self.k, self.lens, self.kept, None, f.table, self.kn, self.vn, self.ring)
        self.before.copy_(f.table)
        self.granted.add_(self.lens)                    # lengths with all of the drafts
        self.lens.add_(self.kept).mul_(~self.done)      # ... with the kept ones
        lynx.lynx_blocks_release(L, B, self.granted, self.lens, f.table, f.stack, f.state)

    def check(self, asked, accept, done):
        """After a step: the plan, the table and stack, and the cache of every sequence."""
        B, bt, H = self.B, self.L.block_tokens, self.H
        old = [x[0].shape[0] for x in self.host]
        starts, plan, before = self.starts.tolist(), [x.tolist() for x in self.plan], self.before.tolist()
        granted = [starts[b + 1] - starts[b] for b in range(B)]
        n = 0
        for b in range(B):
            assert granted[b] in (0, asked[b])
            for i in range(granted[b]):
                p = old[b] + i
                assert [x[n] for x in plan] == [b, p, before[b][p // bt] * bt + p % bt, b * self.k + i]
                n += 1
        assert all(x[n:] == [-1] * (len(x) - n) for x in plan)
        rows = torch.tensor(plan[3][:n], dtype=torch.long)
        if n:
            y, bound = reference(self.qkv[:n, self.Hq:self.Hq + H], self.w[1], self.plan[1][:n], self.f, False, 1.0)
            got = self.kn.view(-1, H, 128).cpu()[rows]
            assert ((got.double() - y).abs() <= bound).all()
            assert torch.equal(self.vn.view(-1, H, 128).cpu()[rows], self.qkv[:n, self.Hq + H:].cpu())
        for b in range(B):
            kept = min(accept[b], granted[b])
            for x, new in zip(range(2), (self.kn, self.vn)):
                self.host[b][x] = torch.cat([self.host[b][x], new[b, :kept].cpu()])[: 0 if done[b] else None]
        lens = [x[0].shape[0] for x in self.host]
        assert self.lens.tolist() == lens
        # every block is on the stack or in one sequence
        table, stack, (free, word) = self.free.table.tolist(), self.free.stack.tolist(), self.free.state.tolist()
        held = [-(-m // bt) for m in lens]
        assert word == 0 and all(row[h:] == [-1] * (len(row) - h) for row, h in zip(table, held))
        assert sorted(stack[:free] + [x for row, h in zip(table, held) for x in row[:h]]) == list(range(self.L.num_blocks))
        # the cache is that of whole sequences
        whole = lynx.KVPool.allocate(self.L, B)
        for b, (k, v) in enumerate(self.host):
            if len(k):
                whole.encode(b, len(k), self.free.table, k.cuda(), v.cuda())
        whole.merge()
        most = max(max(lens), 1)
        back = [[torch.zeros(B, most, H, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2)]
        for pool, out in zip((whole, self.pool), back):
            lynx.lynx_kv_dequant(self.L, B, most, ints([0] * B), self.lens, self.free.table, pool.k_codes, pool.v_codes, pool.meta, *out)
        assert torch.equal(back[0][0], back[1][0]) and torch.equal(back[0][1], back[1][1])
        assert torch.isfinite(self.out[[b for b in range(B) if granted[b] == self.k]]).all()
        return granted


@pytest.mark.parametrize("captured", [False, True])
def test_steps_that_keep_some_drafts(captured):
    B, k, bt = 5, 40, 16
    s = Server(B, k, bt, per=14, n_blocks=34)
    g = torch.Generator().manual_seed(3)
    graph = None
    if captured:
        s.step()  # (asks for nothing)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.step()
    refused = 0
    for i in range(14):
        if i == 0:
            asked, accept, done = [40, 7, 0, 16, 33], [40, 7, 0, 16, 33], [False] * B  # prompts
        else:
            asked = torch.randint(0, k + 1, (B,), generator=g).tolist()
            accept = [int(torch.randint(0, n + 1, (1,), generator=g)) for n in asked]
            done = [i % 4 == 3 and b == i % B for b in range(B)]
        s.qkv.copy_(torch.randn(s.qkv.shape, generator=g))
        for x, y in ((s.asked, asked), (s.accept, accept), (s.done, done)):
            x.copy_(torch.tensor(y))
        note(f"step {i} captured={captured} asked={asked} accept={accept} done={done}")
        graph.replay() if captured else s.step()
        torch.cuda.synchronize()
        granted = s.check(asked, accept, done)
        refused += sum(a > 0 and n == 0 for a, n in zip(asked, granted))
    assert refused


@pytest.mark.parametrize("whole", [True, False])
def test_hierarchical_step_with_its_lse(whole, monkeypatch):
    """The kept drafts' blocks stay, the others' go back; outputs and lse against 64 bits,
    eager and replayed."""
    if not whole:
        monkeypatch.setattr(lynx, "_whole", lambda *args: None)
    lens, Hq, H, bt, k, per = [300, 5, 0, 129], 8, 2, 16, 20, 24
    B, n_blocks, keep = len(lens), 96, [20, 12, 0, 3]
    L = lynx.Layout(num_kv_heads=H, block_tokens=bt, max_blocks_per_seq=per, num_blocks=n_blocks, max_tokens=per * bt)
    free = lynx.FreeBlocks.allocate(L, B)
    granted, starts = ints([0] * B), ints([0] * (B + 1))
    lynx.lynx_blocks_extend(L, B, 300, ints([0] * B), ints(lens), free.table, free.stack, free.state, granted, starts)
    pool, hm = lynx.KVPool.allocate(L, B, codes=False), lynx.HMeta.empty(L, B)
    for b, n in enumerate(lens):
        kk, vv = random_kv(n, H, seed=b)
        lynx.lynx_hkv_encode(L, b, n, free.table, kk.cuda(), vv.cuda(), 255.0, INT4, pool.k_anc, pool.v_anc, None, None, hm)
    start = [x.clone() for x in (free.table, free.stack, free.state)]
    g = torch.Generator().manual_seed(3)
    N = B * k
    qkv, w, f = torch.zeros(N, Hq + 2 * H, 128, dtype=torch.bfloat16, device="cuda"), [None, None], freqs(64)
    d_lens, counts, kept, after, now = ints(lens), ints([k] * B), ints(keep), ints([0] * B), ints([0] * B)
    positions, rows = ints([0] * N), ints([0] * N)
    q, kt, vt, out = (torch.zeros(B, k, h, 128, dtype=torch.bfloat16, device="cuda") for h in (Hq, H, H, Hq))
    lse, ws = torch.zeros(B, k, Hq, device="cuda"), lynx.workspace(L, B, Hq, k, L.max_tokens, tree=False)

    def step():
        lynx.lynx_blocks_extend(L, B, k, d_lens, counts, free.table, free.stack, free.state, granted, starts, None, positions,
                                None, rows)
        lynx.lynx_qk_norm_rope(qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:], positions, rows, *w, EPS, f, True, 1.0, q, kt, vt)
        lynx.lynx_attn_hier(L, B, Hq, k, L.max_tokens, d_lens, free.table, False, pool.k_anc, pool.v_anc, 255.0, INT4, hm, q, kt,
                            vt, out, lse, ws)
        torch.add(d_lens, granted, out=after)
        torch.add(d_lens, kept, out=now)
        lynx.lynx_blocks_release(L, B, after, now, free.table, free.stack, free.state)

    def check():
        torch.cuda.synchronize()
        assert granted.tolist() == [k] * B and positions.tolist() == [n + i for n in lens for i in range(k)]
        ref, bound, ref_lse, lse_bound = attention(L, lens, start[0].cpu(), (pool.k_anc.cpu(), pool.v_anc.cpu()),
                                                   [getattr(hm, x).cpu() for x in lynx._HMETA_NAMES], False, 255.0, INT4, q.cpu(),
                                                   kt.cpu(), vt.cpu())
        assert_inside(out, lse, ref, bound, ref_lse, lse_bound)
        held = [-(-(n + m) // bt) for n, m in zip(lens, keep)]
        table, (left, word) = free.table.tolist(), free.state.tolist()
        assert word == 0 and left == n_blocks - sum(held)
        assert sorted(free.stack.tolist()[:left] + [x for row, h in zip(table, held) for x in row[:h]]) == list(range(n_blocks))
        assert all(row[h:] == [-1] * (per - h) for row, h in zip(table, held))

    def again():
        for x, y in zip((free.table, free.stack, free.state), start):
            x.copy_(y)
        lse.fill_(math.nan)
        out.fill_(math.nan)
        qkv.copy_(torch.randn(qkv.shape, generator=g))
    again()
    note("hierarchical step, eager")
    step()
    check()
    again()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        again()
        note(f"hierarchical step, replay {i}")
        graph.replay()
        check()
