"""Tokens appended to the cache: after any appends its planes and metadata are
those of encoding the whole sequence at once, bit for bit (the oracle's encode
and merge); reading back is fma(code, scale, zero) rounded to BF16."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
from oracle import tree
from paper_2607_01831_amd import inputs, lynx
from tests.gpu_cases import bits, build_cache, note, random_bf16, random_kv
from tests.test_gpu_tree import ATOL, RTOL, random_parents
from tests._util import assert_close

pytestmark = pytest.mark.gpu

PLANES = ("k_anc", "v_anc", "k_res", "v_res", "k_codes", "v_codes")
MARK = 0xA5  # what no append has written


class Grown:
    """Sequences that grow by appends, and their whole K and V."""

    def __init__(self, B, Hkv, capacity, bt=None, seed=0, planes=PLANES):
        self.B, self.Hkv, self.capacity, self.seed = B, Hkv, capacity, seed
        bt = bt or capacity
        per = -(-capacity // bt)
        order = torch.randperm(B * per, generator=torch.Generator().manual_seed(seed)) if per > 1 else torch.arange(B)
        self.table = order.to(torch.int32).view(B, per)
        self.L = lynx.Layout(num_kv_heads=Hkv, block_tokens=bt, max_blocks_per_seq=per, num_blocks=B * per,
                             max_tokens=capacity)
        self.pool = lynx.KVPool.allocate(self.L, B)
        for name in PLANES:
            getattr(self.pool, name).fill_(MARK)
        self.planes = planes
        self.ring = self.pool.open_rows()
        self.ring.fill_(float("nan"))  # needs no initialisation
        kv = [random_kv(capacity, Hkv, seed=seed + 10 + b) for b in range(B)]
        self.k, self.v = [torch.stack(x) for x in zip(*kv)]
        self.lens = [0] * B

    def append(self, counts, max_new=None, path=None, n_src=None, say=None):
        """The next counts[b] tokens of every sequence; rows of k_new past them,
        and those that the path skips, hold NaN."""
        most = max_new if max_new is not None else max(counts)
        n_src = n_src or most
        kn = torch.full((self.B, n_src, self.Hkv, 128), float("nan"), dtype=torch.bfloat16)
        vn = kn.clone()
        for b, c in enumerate(counts):
            for i in range(max(0, min(c, most, self.capacity - self.lens[b]))):
                row = i if path is None else path[b][i]
                kn[b, row], vn[b, row] = self.k[b, self.lens[b] + i], self.v[b, self.lens[b] + i]
        ints = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
        p = None if path is None else ints([list(x) + [-1] * (most - len(x)) for x in path])
        note(f"append {counts[:4]} of {most} behind {self.lens[:4]} bt={self.L.block_tokens}")
        pl = [getattr(self.pool, x) if x in self.planes else None for x in ("k_codes", "v_codes", "k_anc", "v_anc", "k_res",
                                                                          "v_res")]
        lynx.lynx_kv_append(self.L, self.B, most, ints(self.lens), ints(say or counts), p, self.table.cuda(), kn.cuda(),
                            vn.cuda(), self.ring, *pl, self.pool.meta)
        torch.cuda.synchronize()
        self.lens = [n + max(0, min(c, most, self.capacity - n)) for n, c in zip(self.lens, counts)]

    def check(self, lens=None):
        """Everything as encoding the whole sequences gives it, and nothing else touched."""
        lens = lens or self.lens
        OL = oracle.Layout(Hkv=self.Hkv, bt=self.L.block_tokens, max_blocks=self.L.max_blocks_per_seq,
                           max_tokens=self.capacity)
        planes, meta = oracle.encode_batch(OL, lens, self.table.numpy(), [bits(self.k[b, :n]) for b, n in enumerate(lens)],
                                           [bits(self.v[b, :n]) for b, n in enumerate(lens)], self.L.num_blocks)
        for x in "kv":
            planes[x + "_codes"] = oracle.merge(planes[x + "_anc"], planes[x + "_res"])
        written = np.zeros(self.L.num_blocks * self.Hkv * self.L.block_tokens, bool)
        for b, n in enumerate(lens):
            written[oracle.token_rows(OL, self.table.numpy(), b, 0, n).reshape(-1)] = True
        for name in PLANES:
            got = getattr(self.pool, name).cpu().numpy().reshape(len(written), -1)
            ref = np.where(written[:, None] & (name in self.planes), planes[name].reshape(len(written), -1), MARK)
            assert np.array_equal(got, ref), (name, lens)
        for name in ("k_scale", "k_zero", "v_scale", "v_zero"):
            got, ref = getattr(self.pool.meta, name).cpu().numpy(), getattr(meta, name)
            assert np.array_equal(got.view(np.uint32), ref.view(np.uint32)), (name, lens)
        ring = bits(self.ring)
        for b, n in enumerate(lens):
            for t in range(max(0, n // 128 - 1) * 128, n):
                assert np.array_equal(ring[b, t % 256], bits(self.k[b, t])), (b, t)


@pytest.mark.parametrize("B,Hkv,bt", [(1, 1, None), (3, 2, 16), (2, 4, 24), (2, 1, 1), (2, 2, 128), (2, 3, 300)])
def test_any_appends_give_the_whole_encode(B, Hkv, bt):
    g = Grown(B, Hkv, 1500, bt, seed=B)
    r = np.random.default_rng(B)
    steps = [[1] * B, [1, 126, 127][:B], [2] * B, [0, 3, 1][:B], [128] * B, [127, 129, 1][:B], [300, 0, 257][:B],
             [255] * B, [1] * B]
    for counts in steps:
        g.append(counts, max_new=max(max(counts), 1) + int(r.integers(0, 40)))
        g.check()


@pytest.mark.parametrize("first", [0, 1, 127, 128, 129, 200, 256, 300])
@pytest.mark.parametrize("count", [1, 127, 128, 129, 255, 256, 257, 500, 640, 900])
def test_long_appends_from_any_length(first, count):
    """The open group's rows are read while later groups' rows of the same half
    of the ring are written."""
    g = Grown(2, 1, 1280, 16, seed=first)
    if first:
        g.append([first, max(first - 1, 0)])
    g.append([count, count])
    g.check()
    g.append([1, 2])  # from the rows just kept
    g.check()


def test_one_token_at_a_time():
    g = Grown(2, 2, 300, 16)
    g.append([120, 250])
    for _ in range(14):
        g.append([1, 1])
        g.check()


def test_a_path_picks_rows_and_may_repeat_them():
    g = Grown(3, 2, 400, 16)
    g.append([100, 126, 3])
    g.append([3, 5, 0], max_new=9, n_src=20, path=[[2, 7, 19], [0, 1, 5, 6, 18], []])
    g.check()
    # the same row twice: the sequence's tokens are equal there
    n = g.lens[0]
    g.k[0, n + 1], g.v[0, n + 1] = g.k[0, n], g.v[0, n]
    g.append([2, 1, 64], max_new=64, n_src=64, path=[[4, 4], [63], list(range(63, -1, -1))])
    g.check()


def test_a_path_ends_at_its_first_row_that_is_not_there():
    for bad in (-1, 20, 2 ** 31 - 1, -2 ** 31):
        g = Grown(2, 1, 300, 16)
        g.append([125, 60])
        g.append([2, 0], max_new=8, n_src=20, path=[[3, 4, bad, 5, 6], [bad, 0, 0]], say=[5, 3])
        g.check()


def test_counts_and_lengths_out_of_range():
    g = Grown(4, 1, 200, 16)
    g.append([10, 150, 199, 200])
    # negative; past max_new; past the capacity; no room at all
    g.append([-5, 30, 40, 3], max_new=20)
    assert g.lens == [10, 170, 200, 200]
    g.check()
    before = [getattr(g.pool, n).clone() for n in PLANES]
    lens = g.lens
    g.lens = [2 ** 31 - 1, 200, 201, 10 ** 6]  # lengths past the capacity: nothing
    g.append([0, 0, 0, 0], max_new=4, say=[4, 4, 4, 4])
    assert all(torch.equal(x, getattr(g.pool, n)) for x, n in zip(before, PLANES))
    g.lens = lens
    g.check()


@pytest.mark.parametrize("planes", [("k_codes", "v_codes"), ("k_anc", "v_anc"), ("k_res", "v_res"),
                                    ("k_codes", "v_codes", "k_anc", "v_anc")])
def test_planes_that_are_not_kept_are_left_out(planes):
    g = Grown(2, 2, 300, 16, planes=planes)
    for c in ([100, 3], [40, 140]):
        g.append(c)
        g.check()


def test_blocks_outside_the_pool_are_skipped():
    g = Grown(1, 2, 256, 16)
    good = g.table.clone()
    g.table[0, 3], g.table[0, 5] = -1, g.L.num_blocks
    g.append([200])
    lost = [int(good[0, i]) for i in (3, 5)]
    OL = oracle.Layout(Hkv=2, bt=16, max_blocks=16, max_tokens=256)
    planes, _ = oracle.encode_batch(OL, [200], good.numpy(), [bits(g.k[0, :200])], [bits(g.v[0, :200])], 16)
    for name in ("k_anc", "v_anc", "k_res", "v_res"):
        got = getattr(g.pool, name).cpu().numpy().reshape(16, -1)
        assert all((got[i] == MARK).all() for i in lost)
        for i in (int(good[0, j]) for j in (0, 1, 2, 4, 6, 7, 8, 9, 10, 11)):
            assert np.array_equal(got[i], planes[name].reshape(16, -1)[i])


def test_lengths_taken_back():
    """Drafts undone: other tokens from a shorter length on, into the group
    before the open one too."""
    g = Grown(2, 2, 600, 16)
    g.append([300, 270])
    g.append([90, 1])           # 390, 271: open groups 3 and 2
    g.lens = [300, 200]         # the group before the open one; 71 tokens back
    g.k[:, 200:], g.v[:, 200:] = random_bf16(g.k[:, 200:].shape, 3), random_bf16(g.v[:, 200:].shape, 4)
    kept = [random_kv(600, 2, seed=10 + b) for b in range(2)]
    g.k[0, :300], g.v[0, :300] = kept[0][0][:300], kept[0][1][:300]
    g.append([100, 80])
    g.check()


@pytest.mark.parametrize("scale", [0.0, 1e-30, 3e38])
def test_flat_and_extreme_groups(scale):
    g = Grown(1, 1, 300, 16)
    g.k *= scale
    g.v[:, ::3] = 1.5
    g.k[0, :, 0, 7] = -0.0
    for c in ([130], [5]):
        g.append(c)
        g.check()


def test_begin_reads_the_codes_and_appends_go_on_from_them():
    """A cache whose BF16 K is gone: the open group is its read-back values."""
    lens, Hkv = [333, 128, 64, 0], 2
    kv = [random_kv(n, Hkv, seed=n) for n in lens]
    c = build_cache([k for k, _ in kv], [v for _, v in kv], Hkv, bt=16, max_tokens=336)
    ring = c.pool.open_rows()
    note("append_begin")
    lynx.lynx_kv_append_begin(c.L, 4, c.lens_dev(), c.table_dev(), c.pool.k_codes, c.pool.meta, ring)
    torch.cuda.synchronize()
    kc, vc = (oracle.merge(c.planes[x + "_anc"], c.planes[x + "_res"]) for x in "kv")
    whole = []
    for b, n in enumerate(lens):
        K = oracle.dequant("full", c.OL, b, n, c.table.numpy(), kc, vc, c.meta)[0] if n else np.zeros((0, Hkv, 128))
        whole.append(torch.tensor(K).float().bfloat16())
        for t in range(max(0, n // 128 - 1) * 128, n):
            assert_close(ring[b, t % 256].float().cpu().numpy(), K[t], 0.0, 2.0 ** -8 * 1.01, "row")
            whole[b][t] = ring[b, t % 256].cpu()
    more = random_kv(2, Hkv, seed=9)
    new = [x.cuda()[None].expand(4, -1, -1, -1).contiguous() for x in more]
    counts = torch.tensor([2, 0, 2, 0], dtype=torch.int32).cuda()
    c.pool.append(2, c.lens_dev(), counts, None, c.table_dev(), *new, ring)
    torch.cuda.synchronize()
    # the open groups, encoded from the read-back rows and the new tokens
    for b, n in ((0, 333), (2, 64)):
        f = n // 128 * 128
        x = torch.cat([whole[b][f:], more[0]]).float()
        lo, hi = x.amin(0), x.amax(0)
        scale = ((hi - lo) / 255).numpy()
        assert np.array_equal(c.pool.meta.k_scale[b, :, f // 128].cpu().numpy(), scale)


@pytest.mark.parametrize("lens,Hkv,bt", [([300], 1, None), ([1000, 5, 0, 129], 2, 16), ([260, 300], 3, 24), ([700] * 3, 2, 1)])
def test_read_back(lens, Hkv, bt):
    kv = [random_kv(n, Hkv, seed=n) for n in lens]
    c = build_cache([k for k, _ in kv], [v for _, v in kv], Hkv, bt=bt)
    kc, vc = (oracle.merge(c.planes[x + "_anc"], c.planes[x + "_res"]) for x in "kv")
    whole = [oracle.dequant("full", c.OL, b, n, c.table.numpy(), kc, vc, c.meta) if n else (np.zeros((0, Hkv, 128)),) * 2
             for b, n in enumerate(lens)]
    r = np.random.default_rng(1)
    for most in (1, 7, 128, 129, max(lens)):
        starts = [int(r.integers(0, max(n, 1))) for n in lens]
        counts = [min(most, n - s) if n else 0 for n, s in zip(lens, starts)]
        out = [torch.full((len(lens), most, Hkv, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        ints = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
        note(f"dequant {starts} {counts} of {most}")
        lynx.lynx_kv_dequant(c.L, len(lens), most, ints(starts), ints(counts), c.table_dev(), c.pool.k_codes, c.pool.v_codes,
                             c.pool.meta, *out)
        torch.cuda.synchronize()
        for b, (s, n) in enumerate(zip(starts, counts)):
            for o, w in zip(out, whole[b]):
                # one rounding to fp32 (the fma's) and one to BF16
                assert_close(o[b, :n].float().cpu().numpy(), w[s:s + n], 0.0, 2.0 ** -8 + 2.0 ** -23, "values")
                assert (o[b, n:] == 7).all()


@pytest.mark.parametrize("Hkv", [4, 6, 8, 12, 16])
def test_read_back_many_heads(Hkv):
    test_read_back([300, 77], Hkv, 16)


def test_read_back_of_more_rows_than_a_grid_holds():
    # 8 heads: workgroups of 8 rows, 65535 of them a launch
    T, Hkv, first = 530_000, 8, 3
    L = lynx.Layout(num_kv_heads=Hkv, block_tokens=T, max_blocks_per_seq=1, num_blocks=1, max_tokens=T)
    g = torch.Generator("cuda").manual_seed(1)
    codes = [torch.randint(0, 256, (Hkv, T, 128), dtype=torch.uint8, device="cuda", generator=g) for _ in range(2)]
    meta = lynx.Meta.empty(L, 1)
    for x in (meta.k_scale, meta.k_zero, meta.v_scale, meta.v_zero):
        x.copy_(torch.randn(x.shape, device="cuda", generator=g))
    out = [torch.full((T - first, Hkv, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ints = lambda x: torch.tensor([x], dtype=torch.int32).cuda()  # noqa: E731
    note(f"dequant {T - first} rows")
    lynx.lynx_kv_dequant(L, 1, T - first, ints(first), ints(T - first), ints(0), *codes, meta, *out)
    torch.cuda.synchronize()
    for at in (first, 2 ** 18, 65535 * 8 - 500, T - 1000):
        t = torch.arange(at, at + 1000, device="cuda")
        ks, kz = (x.view(Hkv, -1, 128)[:, t // 128].double() for x in (meta.k_scale, meta.k_zero))
        vs, vz = (x.view(Hkv, T, 1)[:, t].double() for x in (meta.v_scale, meta.v_zero))
        for o, c, sc, z in ((out[0], codes[0], ks, kz), (out[1], codes[1], vs, vz)):
            want = (c[:, t].double() * sc + z).transpose(0, 1)
            assert_close(o[t - first].float().cpu().numpy(), want.cpu().numpy(), 0.0, 2.0 ** -8 + 2.0 ** -23, "values")


def test_read_back_out_of_range():
    kv = random_kv(200, 2, seed=1)
    c = build_cache([kv[0]] * 5, [kv[1]] * 5, 2, bt=16)
    c.table[4, 0] = -1
    out = [torch.full((5, 40, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    starts = torch.tensor([-1, 2 ** 31 - 1, 190, 100, 10], dtype=torch.int32).cuda()
    counts = torch.tensor([40, 40, 2 ** 31 - 1, -3, 12], dtype=torch.int32).cuda()
    lynx.lynx_kv_dequant(c.L, 5, 40, starts, counts, c.table_dev(), c.pool.k_codes, c.pool.v_codes, c.pool.meta, *out)
    torch.cuda.synchronize()
    for o in out:
        touched = (o != 7).flatten(2).any(2).cpu()
        want = torch.zeros(5, 40, dtype=torch.bool)
        want[2, :10] = True   # up to the capacity of 200
        want[4, 6:12] = True  # block 0's tokens are skipped
        assert torch.equal(touched, want)


def test_blocks_past_four_gigabytes():
    """The same calls with the sequence in the first and in the last blocks of a
    pool whose planes are larger than 2^32 bytes: the same bits."""
    T, Hkv, bt, n, blocks = 1000, 8, 16, 40, 270_000
    per = -(-(T + 64) // bt)
    L = lynx.Layout(num_kv_heads=Hkv, block_tokens=bt, max_blocks_per_seq=per, num_blocks=blocks, max_tokens=T + 64)
    assert L.plane_bytes(128) > 2 ** 32 + per * bt * Hkv * 128
    planes = [torch.empty(L.plane_bytes(128), dtype=torch.uint8, device="cuda") for _ in range(2)]
    k, v = (x[None].cuda() for x in random_kv(T, Hkv, seed=3))
    q, kn, vn = (random_bf16((1, n, h, 128), 5 + i).cuda() for i, h in enumerate((32, Hkv, Hkv)))
    ints = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    parents = ints(random_parents(1, n, seed=4).tolist())
    f = lynx.load().lynx_internal_verify_tree
    P, I = ctypes.c_void_p, ctypes.c_int32
    f.argtypes = [P, I, I, I, I, P, P, P, P, P, P, P, P, P, P, P, ctypes.c_size_t, P, I]
    results = []
    for first in (0, blocks - per):
        meta = lynx.Meta.empty(L, 1)
        table = torch.arange(first, first + per, dtype=torch.int32, device="cuda").view(1, per)
        ring = torch.zeros(1, 256, Hkv, 128, dtype=torch.bfloat16, device="cuda")
        note(f"blocks from {first}")
        lynx.lynx_kv_append(L, 1, T, ints([0]), ints([T]), None, table, k, v, ring, *planes, None, None, None, None, meta)
        back = [torch.zeros(1, T, Hkv, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        lynx.lynx_kv_dequant(L, 1, T, ints([0]), ints([T]), table, *planes, meta, *back)
        again = torch.zeros_like(ring)
        lynx.lynx_kv_append_begin(L, 1, ints([T]), table, planes[0], meta, again)
        torch.cuda.synchronize()
        got = [*back, again, ring, meta.k_scale, meta.v_zero]
        lens, ws = ints([T]), torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
        for wide in (0, 1, 2):
            out = torch.zeros_like(q)
            dev = [lens, table, *planes, q, kn, vn, parents, out, ws]
            lp, tp, kp, vp, qp, knp, vnp, pp, op, wp = (x.data_ptr() for x in dev)
            assert f(ctypes.byref(L.c()), 1, 32, n, T, lp, tp, kp, vp, ctypes.byref(meta.c()), qp, knp, vnp, pp, op, wp,
                     ws.nbytes, torch.cuda.current_stream().cuda_stream, wide) == 0
            torch.cuda.synchronize()
            got.append(out)
        results.append([x.cpu() for x in got])
    for x, y in zip(*results):
        assert torch.equal(x, y)
    # and what was read back is what was written: half a code's step (largest
    # scale) and the rounding to BF16, 2^-8 of the value, which is at most the
    # written one and that half step
    half, written = results[0][4].max().item() / 2, k.cpu().float()
    error = (results[0][0].float() - written).abs()
    assert (error <= half * 1.001 + (written.abs() + half) * 2.0 ** -8).all()


def step_inputs(B, n, Hq, Hkv, V, seed):
    q, kn, vn = (random_bf16((B, n, h, 128), seed + i) for i, h in enumerate((Hq, Hkv, Hkv)))
    r = np.random.default_rng(seed)
    logits = np.round(r.standard_normal((B, n + 1, V)) * 8).astype(np.float32)
    parents = random_parents(B, n, seed, chain=0.7)
    tokens = np.zeros((B, n), np.int32)
    for b in range(B):
        for i in range(n):
            tokens[b, i] = tree.choice_greedy(logits[b, parents[b, i] + 1]) if r.random() < 0.8 else r.integers(0, V)
    return q, kn, vn, logits, parents, tokens


@pytest.mark.parametrize("captured", [False, True])
def test_the_operators_together(captured):
    """Decoding steps as a server makes them: a tree is verified over the cache,
    its longest agreeing path kept, and the kept tokens' K and V appended, whose
    codes the next step's verification reads; eager, and as one graph."""
    B, Hkv, Hq, n, V, capacity = 3, 2, 8, 10, 700, 700
    g = Grown(B, Hkv, capacity, 16, seed=20)
    g.append([250, 127, 0], max_new=250)
    lens = torch.tensor(g.lens, dtype=torch.int32, device="cuda")
    table = g.table.cuda()
    dev = dict(q=torch.zeros(B, n, Hq, 128, dtype=torch.bfloat16), kn=torch.zeros(B, n, Hkv, 128, dtype=torch.bfloat16),
               vn=torch.zeros(B, n, Hkv, 128, dtype=torch.bfloat16), logits=torch.zeros(B, n + 1, V),
               parents=torch.zeros(B, n, dtype=torch.int32), tokens=torch.zeros(B, n, dtype=torch.int32))
    dev = {k: x.cuda() for k, x in dev.items()}
    out = torch.empty_like(dev["q"])
    accepted, nxt = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    path = torch.zeros(B, n, dtype=torch.int32, device="cuda")
    ws, wt = lynx.workspace(g.L, B, Hq, n, capacity), lynx.spec_tree_workspace(B, n, V)

    def step():
        lynx.lynx_attn_verify_tree(g.L, B, Hq, n, capacity, lens, table, g.pool.k_codes, g.pool.v_codes, g.pool.meta, dev["q"],
                                   dev["kn"], dev["vn"], dev["parents"], out, ws)
        lynx.lynx_spec_accept_tree_greedy(dev["logits"], dev["tokens"], dev["parents"], accepted, path, nxt, wt)
        g.pool.append(n, lens, accepted, path, table, dev["kn"], dev["vn"], g.ring)
        lens.add_(accepted)

    graph = None
    if captured:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    OL = oracle.Layout(Hkv=Hkv, bt=16, max_blocks=g.L.max_blocks_per_seq, max_tokens=capacity)
    for turn in range(6):
        q, kn, vn, logits, parents, tokens = step_inputs(B, n, Hq, Hkv, V, 100 + turn)
        for name, x in zip(("q", "kn", "vn", "logits", "parents", "tokens"),
                           (q, kn, vn, torch.as_tensor(logits), torch.as_tensor(parents), torch.as_tensor(tokens))):
            dev[name].copy_(x)
        codes = [x.cpu().numpy() for x in (g.pool.k_codes, g.pool.v_codes)]
        m = g.pool.meta
        meta = oracle.Meta(*(x.cpu().numpy().copy() for x in (m.k_scale, m.k_zero, m.v_scale, m.v_zero)))
        note(f"step {turn} lens={g.lens}")
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        assert_close(out.float().cpu().numpy(),
                     tree.verify_tree(OL, Hq, g.lens, g.table.numpy(), *codes, meta, bits(q), bits(kn), bits(vn), parents),
                     ATOL, RTOL, "verification")
        a, p, t = tree.accept_tree(logits, tokens, parents)
        for got, ref in ((accepted, a), (path, p), (nxt, t)):
            assert np.array_equal(got.cpu().numpy(), ref)
        for b in range(B):
            for i in range(a[b]):
                g.k[b, g.lens[b] + i], g.v[b, g.lens[b] + i] = kn[b, p[b, i]], vn[b, p[b, i]]
        g.lens = [x + int(y) for x, y in zip(g.lens, a)]
        assert lens.tolist() == g.lens
        g.check()
    assert sum(g.lens) > 250 + 127
