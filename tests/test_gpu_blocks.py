"""The blocks of a step, entry by entry against a plain walk over the batch:
lengths, block sizes, refusals for want of blocks or rows, what is left alone,
blocks given back, batches of one to thousands, graphs."""
import numpy as np
import pytest
import torch

from paper_2607_01831_amd import lynx
from tests.gpu_cases import note

pytestmark = pytest.mark.gpu


def plan(lens, counts, table, stack, n_free, bt, n_src, max_rows, capacity, n_blocks):
    """The extend call in Python; table and the count change in place."""
    B = len(lens)
    out = dict(granted=[0] * B, starts=[0], **{x: [-1] * max_rows for x in ("seq_of", "positions", "slots", "rows")})
    asked = tokens = n = taken = 0
    for b in range(B):
        T = min(max(lens[b], 0), capacity)
        c = min(max(counts[b], 0), n_src, capacity - T)
        held, end = -(-T // bt), -(-(T + c) // bt)
        first = asked  # the stack's entries by what was asked before, refused or not
        asked += end - held
        tokens += c
        if (end == held or asked <= n_free) and tokens <= max_rows:
            out["granted"][b] = c
            for j in range(held, end):
                table[b, j] = stack[n_free - 1 - first - (j - held)]
            taken += end - held
            for i in range(c):
                p = T + i
                blk = int(table[b, p // bt])
                out["seq_of"][n], out["positions"][n], out["rows"][n] = b, p, b * n_src + i
                out["slots"][n] = blk * bt + p % bt if 0 <= blk < n_blocks else -1
                n += 1
        out["starts"].append(n)
    return out, n_free - taken


def drop(lens, keep, table, stack, n_free, bt, capacity, n_blocks):
    back = []
    for b in range(len(lens)):
        T = min(max(lens[b], 0), capacity)
        k = min(max(keep[b], 0), T)
        for j in range(-(-k // bt), -(-T // bt)):
            back.append(table[b, j])
            table[b, j] = -1
    for n, x in enumerate(back):
        at = n_free + len(back) - 1 - n
        if at < n_blocks:
            stack[at] = x
    return min(n_free + len(back), n_blocks)


class Pool:
    def __init__(self, lens, bt, per, free, seed=0, n_blocks=None):
        B, r = len(lens), np.random.default_rng(seed)
        held = [-(-n // bt) for n in lens]
        self.n_blocks = n_blocks or max(sum(held) + free, 1)
        ids = r.permutation(self.n_blocks).astype(np.int32)
        self.table = np.full((B, per), -1, np.int32)
        at = 0
        for b, n in enumerate(held):
            self.table[b, :n] = ids[at:at + n]
            at += n
        self.stack = np.full(self.n_blocks, -9, np.int32)
        self.stack[:free] = ids[at:at + free]
        self.free, self.bt, self.capacity, self.lens = free, bt, per * bt, list(lens)
        self.L = lynx.Layout(num_kv_heads=1, block_tokens=bt, max_blocks_per_seq=per, num_blocks=self.n_blocks,
                             max_tokens=per * bt)
        dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
        self.d_table, self.d_stack = dev(self.table), dev(self.stack)
        self.d_state = torch.tensor([free, 0], dtype=torch.int32).cuda()

    def ints(self, x):
        return torch.tensor(x, dtype=torch.int32).cuda()

    def same(self):
        assert self.d_state.tolist() == [self.free, 0]
        assert np.array_equal(self.d_table.cpu().numpy(), self.table)
        assert np.array_equal(self.d_stack.cpu().numpy(), self.stack)

    def extend(self, counts, n_src, max_rows, names=("seq_of", "positions", "slots", "rows"), lens=None):
        B = len(self.lens)
        lens = self.lens if lens is None else lens
        note(f"blocks_extend B={B} bt={self.bt} n_src={n_src} rows={max_rows} free={self.free}")
        got = {x: torch.full((max_rows,), -77, dtype=torch.int32, device="cuda") for x in names}
        granted, starts = (torch.full((n,), -77, dtype=torch.int32, device="cuda") for n in (B, B + 1))
        lynx.lynx_blocks_extend(self.L, B, n_src, self.ints(lens), self.ints(counts), self.d_table, self.d_stack,
                                self.d_state, granted, starts, *(got.get(x) for x in ("seq_of", "positions", "slots", "rows")))
        want, self.free = plan(lens, counts, self.table, self.stack, self.free, self.bt, n_src, max_rows, self.capacity,
                               self.n_blocks)
        for x, t in {**got, "granted": granted, "starts": starts}.items():
            assert t.tolist() == want[x], x
        self.same()
        self.lens = [n + g for n, g in zip(lens, want["granted"])]
        return want

    def release(self, keep):
        note(f"blocks_release B={len(self.lens)} bt={self.bt}")
        lynx.lynx_blocks_release(self.L, len(self.lens), self.ints(self.lens), self.ints(keep), self.d_table, self.d_stack,
                                 self.d_state)
        self.free = drop(self.lens, keep, self.table, self.stack, self.free, self.bt, self.capacity, self.n_blocks)
        self.same()
        self.lens = [min(max(k, 0), n) for k, n in zip(keep, self.lens)]


@pytest.mark.parametrize("bt", [1, 5, 16, 128])
@pytest.mark.parametrize("B,most", [(1, 1), (1, 300), (3, 70), (64, 9), (255, 3), (256, 4), (257, 5), (1030, 2), (2100, 3),
                                    (20000, 2)])
def test_extend_and_release(B, most, bt):
    r = np.random.default_rng(B * 131 + bt)
    lens = r.integers(0, 200, B).tolist()
    counts = r.integers(-1, most + 2, B).tolist()
    p = Pool(lens, bt, -(-(200 + most) // bt) + 1, free=B * (most + 1), seed=B)
    want = p.extend(counts, most, B * most)
    assert want["granted"] == [min(max(c, 0), most) for c in counts]
    # drafts dropped: some kept, some sequences done
    p.release([n - int(r.integers(0, 5)) if i % 4 else 0 for i, n in enumerate(p.lens)])
    p.extend(r.integers(0, most + 1, B).tolist(), most, B * most + 3)


def test_release_restores_the_stack():
    p = Pool([10, 0, 33], 16, 8, free=9, seed=4)
    stack, table = p.stack.copy(), p.table.copy()
    before = list(p.lens)
    p.extend([40, 17, 1], 40, 58)
    assert p.free < 9
    p.release(before)
    assert np.array_equal(p.stack, stack) and np.array_equal(p.table, table) and p.free == 9


@pytest.mark.parametrize("free", [0, 1, 2, 3, 4, 7])
def test_refused_for_want_of_blocks(free):
    """The first that does not fit and later ones that need a block get nothing; ones
    that need none get their tokens."""
    p = Pool([16, 3, 0, 15, 32, 5], 16, 5, free=free, seed=free)
    p.extend([1, 13, 33, 1, 20, 0], 40, 200)


@pytest.mark.parametrize("rows", [0, 1, 5, 6, 40, 107])
def test_refused_for_want_of_rows(rows):
    p = Pool([16, 3, 0, 15], 16, 5, free=50)
    p.extend([5, 1, 33, 1], 40, rows)


def test_capacity_and_clamped_arguments():
    p = Pool([60, 64, 0], 16, 4, free=20)
    p.extend([10, 3, 2000], 500, 700)                    # 64 tokens hold them
    q = Pool([60, 64, 0], 16, 4, free=20)
    q.extend([1, 1, 1], 2, 8, lens=[-5, 2 ** 31 - 1, 0])  # lengths clamped
    q = Pool([20, 20], 16, 4, free=5)
    q.d_state[0] = 2 ** 31 - 1                           # more than there are blocks
    q.free = q.n_blocks
    q.extend([3, 3], 4, 8)


def test_none_arrays_and_ids_outside_the_pool():
    p = Pool([20, 30], 16, 4, free=5)
    p.table[0, 1] = 10 ** 6
    p.stack[p.free - 1] = -4
    p.d_table, p.d_stack = torch.from_numpy(p.table).cuda(), torch.from_numpy(p.stack).cuda()
    p.extend([14, 9], 16, 32)  # both stand in slots as -1
    for names in ((), ("slots",), ("rows", "positions")):
        q = Pool([20, 30], 16, 4, free=5)
        q.extend([14, 9], 16, 32, names=names)


def test_release_past_the_stacks_end():
    p = Pool([40, 40], 16, 4, free=4, n_blocks=10)
    p.d_state[0] = 8
    p.free = 8
    p.release([0, 17])


def test_many_rows_and_graph():
    """Thousands of rows over many workgroups; a captured step on changing lengths."""
    r = np.random.default_rng(5)
    B, most = 300, 900
    p = Pool(r.integers(0, 3000, B).tolist(), 16, 300, free=17000, seed=2)
    p.extend(r.integers(0, most, B).tolist(), most, B * most)
    p.release([n // 2 for n in p.lens])
    lens, counts = p.ints(p.lens), p.ints([7] * B)
    outs = [torch.empty(n, dtype=torch.int32, device="cuda") for n in (B, B + 1, 7 * B, 7 * B, 7 * B, 7 * B)]

    def step():
        lynx.lynx_blocks_extend(p.L, B, 7, lens, counts, p.d_table, p.d_stack, p.d_state, *outs)
        lens.add_(outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want, p.free = plan(p.lens, [7] * B, p.table, p.stack, p.free, 16, 7, 7 * B, p.capacity, p.n_blocks)
        p.lens = [n + g for n, g in zip(p.lens, want["granted"])]
        for x, t in zip(("granted", "starts", "seq_of", "positions", "slots", "rows"), outs):
            assert t.tolist() == want[x], x
        p.same()
        assert lens.tolist() == p.lens


def test_streams():
    pools = [Pool([100 * i, 5], 16, 40, free=60, seed=i) for i in (1, 2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for p, s in zip(pools, streams):
            with torch.cuda.stream(s):
                p.extend([30, 3], 30, 60)
                p.release([p.lens[0] - 20, p.lens[1]])
