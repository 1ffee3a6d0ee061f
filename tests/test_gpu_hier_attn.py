"""Attention over the hierarchical codec's cache against 64 bits: every variant of
the codec from 4-bit planes and merged codes, head layouts, lengths around the
codec's chunks and pages and the kernel's units, block sizes that chunks straddle,
tails, empty sequences, bad block ids, what lies behind a sequence, extreme ranges,
streams, graphs, shared workspaces and pools past 2^32 bytes."""
import math

import numpy as np
import pytest
import torch

from paper_2607_01831_amd import inputs, lynx
from tests.gpu_cases import note, random_bf16, random_kv
from tests.hier_ref import BIASED, CENTRED, INT4, attention, level_table, side

pytestmark = pytest.mark.gpu


class Case:
    """A cache that lynx_hkv_encode filled, ragged and paged (bt None: contiguous)."""

    def __init__(self, lens, Hkv, variant, full=False, alpha=255.0, bt=None, seed=0, kv=None, spare=0):
        self.lens, self.variant, self.full, self.alpha = list(lens), variant, full, alpha
        B, most = len(lens), max(max(lens), 1) + spare
        if bt is None:
            self.table, blocks, bt = torch.arange(B, dtype=torch.int32).view(B, 1), B, most
        else:
            self.table, blocks = inputs.paged_block_table(torch.tensor([n + spare for n in lens]), bt, seed)
        self.L = lynx.Layout(num_kv_heads=Hkv, block_tokens=bt, max_blocks_per_seq=self.table.shape[1],
                             num_blocks=max(blocks, 1), max_tokens=most)
        self.pool, self.hm = lynx.KVPool.allocate(self.L, B), lynx.HMeta.empty(self.L, B)
        self.dev_table, self.dev_lens = self.table.cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda()
        for b, n in enumerate(lens):
            k, v = kv[b] if kv else random_kv(n, Hkv, seed=seed + 17 * b)
            lynx.lynx_hkv_encode(self.L, b, n, self.dev_table, k.cuda(), v.cuda(), alpha, variant, self.pool.k_anc,
                                 self.pool.v_anc, self.pool.k_res, self.pool.v_res, self.hm)
        if full:
            self.pool.merge()
        self.planes = (self.pool.k_codes, self.pool.v_codes) if full else (self.pool.k_anc, self.pool.v_anc)

    def host(self):
        return tuple(p.cpu() for p in self.planes), [getattr(self.hm, f).cpu() for f in lynx._HMETA_NAMES]

    def call(self, q, kt=None, vt=None, most=None, ws=None, out=None, lse=None, stream=None):
        B, k, Hq, _ = q.shape
        most = max(self.lens) if most is None else most
        out = torch.full_like(q, math.nan) if out is None else out
        lse = torch.full((B, k, Hq), math.nan, device="cuda") if lse is None else lse
        ws = lynx.workspace(self.L, B, Hq, k, most, tree=False) if ws is None else ws
        lynx.lynx_attn_hier(self.L, B, Hq, k, most, self.dev_lens, self.dev_table, self.full, *self.planes, self.alpha,
                            self.variant, self.hm, q, kt, vt, out, lse, ws, stream)
        return out, lse

    def queries(self, Hq, k, n_tail, seed=5):
        B, H = len(self.lens), self.L.num_kv_heads
        tail = [random_bf16((B, n_tail, H, 128), seed + i) for i in (1, 2)] if n_tail else [None, None]
        return random_bf16((B, k, Hq, 128), seed), *tail

    def check(self, Hq, k=1, n_tail=0, seed=5, q=None, **kw):
        q0, kt, vt = self.queries(Hq, k, n_tail, seed)
        q = q0 if q is None else q
        note(f"attn_hier lens={self.lens[:4]} B={len(self.lens)} Hkv={self.L.num_kv_heads} Hq={Hq} k={k} tail={n_tail} "
             f"bt={self.L.block_tokens} variant={self.variant} full={self.full} alpha={self.alpha}")
        dev = lambda x: None if x is None else x.cuda()  # noqa: E731
        out, lse = self.call(q.cuda(), dev(kt), dev(vt), **kw)
        torch.cuda.synchronize()
        planes, hm = self.host()
        ref, bound, ref_lse, lse_bound = attention(self.L, self.lens, self.table, planes, hm, self.full, self.alpha,
                                                   self.variant, q, kt, vt)
        assert_inside(out, lse, ref, bound, ref_lse, lse_bound)
        return out, lse


def assert_inside(out, lse, ref, bound, ref_lse, lse_bound):
    got = out.double().cpu()
    off = (got - ref).abs()
    assert torch.isfinite(got).all()
    assert (off <= bound).all(), f"off by {off.max():.3e}, {(off / bound).max():.2f} of the bound"
    l = lse.double().cpu()
    empty = ref_lse == -math.inf
    assert (l[empty] == -math.inf).all() and (got[empty] == 0).all()
    assert ((l - ref_lse).abs()[~empty] <= lse_bound[~empty]).all()


FORMS = [(BIASED, False), (BIASED, True), (CENTRED, False), (CENTRED, True), (INT4, False)]


@pytest.mark.parametrize("variant,full", FORMS)
def test_reference_is_the_codec(variant, full):
    """The reference's keys and values, rounded to BF16, are lynx_hkv_dequant's but
    for its fp32 products (a value in a few hundred, by a step)."""
    c = Case([300], 2, variant, full, seed=3)
    ko, vo = (torch.empty(300, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lynx.lynx_hkv_dequant(c.L, 0, 300, c.dev_table, full, *c.planes, c.alpha, variant, c.hm, ko, vo)
    planes, hm = c.host()
    for h in range(2):
        for got, plane, m in ((ko, planes[0], hm[:4]), (vo, planes[1], hm[4:])):
            x, _ = side(plane, *m, c.L, c.table, 0, h, 300, full, level_table(c.alpha, variant, full))
            top = (m[0].abs() + m[1].abs()).max().item()
            assert ((got[:, h].double().cpu() - x).abs() <= 2.0 ** -8 * x.abs() + 2.0 ** -21 * top).all()


@pytest.mark.parametrize("variant,full", FORMS)
@pytest.mark.parametrize("T,Hkv,G,bt", [(1, 1, 1, None), (2, 2, 4, 16), (31, 1, 3, None), (32, 2, 4, 24), (33, 1, 8, 32),
                                        (127, 4, 2, 16), (257, 2, 7, 48), (513, 1, 16, 7), (1000, 2, 4, None)])
def test_decode_lengths(variant, full, T, Hkv, G, bt):
    Case([T], Hkv, variant, full, bt=bt, seed=T).check(Hkv * G)


@pytest.mark.parametrize("variant,full", FORMS)
@pytest.mark.parametrize("lens,Hkv,G,k,tail,bt", [
    ((300, 0, 1, 65), 2, 4, 1, 0, 16), ((300, 0, 1, 65), 2, 4, 1, 1, 16), ((40, 700), 2, 4, 1, 64, None),
    ((130, 0), 2, 4, 4, 4, 16), ((511, 513, 512), 1, 7, 5, 9, 48), ((96, 2000), 2, 8, 3, 0, None),
    ((90,), 1, 2, 64, 64, 5), ((600, 33), 1, 1, 33, 40, 32), ((1025,), 2, 20, 1, 3, 64), ((70,), 1, 40, 1, 0, None)])
def test_queries_and_tails(variant, full, lens, Hkv, G, k, tail, bt):
    Case(lens, Hkv, variant, full, bt=bt, seed=sum(lens)).check(Hkv * G, k, tail)


@pytest.mark.parametrize("B,most,bt,G,k,tail,full", [(70, 900, 16, 4, 1, 0, False), (20, 3000, 32, 2, 1, 5, False),
                                                     (9, 5000, None, 4, 6, 6, True), (66, 1200, 24, 1, 2, 3, True)])
def test_batches_of_many_units(B, most, bt, G, k, tail, full):
    """More units than workgroups: shares that cross sequences, empty ones between."""
    r = np.random.default_rng(B)
    lens = [0 if i % 11 == 4 else int(r.integers(1, most)) for i in range(B)]
    Case(lens, 8, CENTRED if full else INT4, full, bt=bt, seed=B).check(8 * G, k, tail)


RAGGED = (0, 1, 129, 4000, 7000, 513, 2900, 8000, 128, 64, 5000, 3100, 700, 2500, 4500, 1)


@pytest.mark.parametrize("lens,G,k,tail,bt", [
    (RAGGED, 4, 1, 0, 16), (RAGGED, 4, 1, 7, 16), (RAGGED[::-1], 2, 3, 4, 32), (RAGGED, 4, 5, 0, 48),
    ((12000, 25000), 4, 2, 2, None), ((33000,), 4, 1, 0, None), ((33000,), 2, 2, 3, 16),
    ((0, 36001), 4, 1, 0, 16), ((9000,) + tuple(range(400, 778, 6)), 2, 1, 1, 16),
    ((512,) * 63 + (3000,), 2, 2, 2, 64), ((1100,) * 22 + (0,) * 42, 4, 1, 0, 16)])
def test_shares_cut_inside_sequences(lens, G, k, tail, bt):
    """More units than workers: shares of whole groups, of one sequence or of many."""
    Case(lens, 8, INT4, bt=bt, seed=len(lens)).check(8 * G, k, tail)


@pytest.mark.parametrize("variant,full", FORMS)
@pytest.mark.parametrize("lens,Hkv,G,k,tail,bt", [((31, 0, 700), 2, 4, 3, 5, 16), ((130, 97), 2, 8, 9, 9, 48),
                                                  ((513,), 1, 5, 64, 64, 24), ((64, 1500), 1, 7, 20, 0, None)])
def test_rows_of_many_tiles(variant, full, lens, Hkv, G, k, tail, bt):
    """Fewer rows than a workgroup's, its number, and more."""
    Case(lens, Hkv, variant, full, bt=bt, seed=sum(lens)).check(Hkv * G, k, tail)


@pytest.mark.parametrize("alpha", [1e-38, 1e-5, 9e-5, 1.1e-4, 1.0, 15.0, 1e4, 1e30])
def test_alpha(alpha):
    for variant, full in FORMS:
        Case([150], 1, variant, full, alpha=alpha, seed=8).check(4)


def test_long_context_and_outlier_channels():
    k, v = random_kv(40000, 1, seed=4, outlier_cols=3, mult=30.0)
    Case([40000], 1, INT4, seed=4, kv=[(k, v + 3.0)]).check(8, 2, 2)


@pytest.mark.parametrize("k_exp,q_exp,v_exp", [(60, -62, 0), (-60, 58, 80), (100, -100, -100), (-90, 90, 100), (6, 0, 110)])
def test_ranges(k_exp, q_exp, v_exp):
    """Powers of two on K, V and the queries pass through."""
    k, v = random_kv(290, 2, seed=9, outlier_cols=1)
    q = random_bf16((1, 3, 8, 128), 6)
    kv = [((k.float() * 2.0 ** k_exp).bfloat16(), (v.float() * 2.0 ** v_exp).bfloat16())]
    c = Case([290], 2, CENTRED, True, seed=9, kv=kv)
    c.check(8, 3, q=(q.float() * 2.0 ** (q_exp - (6 if k_exp == 6 else 0))).bfloat16())


def test_pages_of_other_ranges():
    """K and V whose size changes from page to page, both ways."""
    k, v = (x.float() for x in random_kv(256 * 6 + 40, 1, seed=12))
    scale = torch.tensor([1.0, 2.0 ** 12, 2.0 ** -9, 2.0 ** 13, 1.0, 2.0 ** -12, 2.0])[torch.arange(len(k)) // 256].view(-1, 1, 1)
    kv = [((k * scale * 2.0 ** -12).bfloat16(), (v * scale).bfloat16())]
    for G, n in ((1, 1), (4, 8)):
        Case([len(k)], 1, INT4, seed=12, kv=kv).check(G, n, n)


def test_zero_cache_and_constant_channels():
    z = torch.zeros(70, 1, 128, dtype=torch.bfloat16)
    Case([70], 1, INT4, kv=[(z, z)]).check(4)
    Case([70], 1, CENTRED, True, kv=[(z + 1.5, z - 2.0)]).check(4, 2, 2)
    for k in (1, 9):  # queries of zeros too: every score is 0, what is masked is not
        Case([70], 1, INT4, kv=[(z, z + 1.0)]).check(4, k, q=torch.zeros(1, k, 4, 128, dtype=torch.bfloat16))


def test_bad_block_ids_poison_their_sequence_alone():
    c = Case([100, 60, 200], 2, INT4, bt=16, seed=2)
    q, _, _ = c.queries(8, 1, 0)
    good, _ = c.call(q.cuda())
    for bad in (-1, c.L.num_blocks, 2 ** 31 - 1, -2 ** 31):
        for at in (0, 3):
            c.dev_table = c.table.clone().cuda()
            c.dev_table[1, at] = bad
            out, lse = c.call(q.cuda())
            assert torch.isnan(out[1]).all() and torch.isnan(lse[1]).all()
            assert torch.equal(out[0], good[0]) and torch.equal(out[2], good[2])
    c.dev_table = c.table.clone().cuda()
    c.dev_table[1, 4:] = -7  # behind the sequence: not read
    assert torch.equal(c.call(q.cuda())[0], good)


@pytest.mark.parametrize("bt", [None, 16, 24])
def test_what_lies_behind_a_sequence_is_not_read(bt):
    """Rows, chunks and pages past the length, and other sequences' NaN, change nothing."""
    c = Case([77, 290], 2, CENTRED, True, bt=bt, seed=6, spare=300)
    q, kt, vt = (x.cuda() for x in c.queries(8, 2, 3))
    good, good_lse = c.call(q, kt, vt)
    for f in lynx._HMETA_NAMES:
        per = 256 if f[2] == "g" else 32
        for b, n in enumerate(c.lens):
            getattr(c.hm, f)[b, :, -(-n // per):] = math.nan
    rows = [p.view(-1, 128) for p in c.planes]
    t = torch.arange(c.L.max_tokens)
    for b, n in enumerate(c.lens):
        behind = t[(t >= n) & (t // c.L.block_tokens < c.table.shape[1])]
        block = c.table[b].long()[behind // c.L.block_tokens]
        for h in range(2):
            at = ((block * 2 + h) * c.L.block_tokens + behind % c.L.block_tokens)[block >= 0].cuda()
            for p in rows:
                p[at] = 0x7F
    out, lse = c.call(q, kt, vt)
    assert torch.equal(out, good) and torch.equal(lse, good_lse)
    c.hm.k_mu[1, :, 0] = math.nan
    out, lse = c.call(q, kt, vt)
    assert torch.equal(out[0], good[0]) and torch.isnan(out[1]).all() and torch.isnan(lse[1]).all()


def test_tail_tokens_not_seen_change_nothing():
    c = Case([50], 1, INT4)
    q, kt, vt = (x.cuda() for x in c.queries(4, 5, 9))
    good, _ = c.call(q, kt, vt)
    kt[:, 5 + 2:], vt[:, 5 + 2:] = math.nan, math.inf  # query i sees tokens 0 .. 4 + i
    out, _ = c.call(q, kt, vt)
    assert torch.equal(out[:, :3], good[:, :3]) and torch.isnan(out[:, 3:]).all()


def test_most_is_a_bound():
    """max_seq_len above the lengths changes no result beyond rounding; lengths past
    it, or negative, are clamped."""
    c = Case([300, 40], 2, INT4, bt=16, spare=2000)
    q, _, _ = c.queries(8, 1, 0)
    c.check(8, most=c.L.max_tokens)
    c.dev_lens = torch.tensor([10 ** 9, -5], dtype=torch.int32).cuda()
    out, lse = c.call(q.cuda(), most=300)
    c.lens = [300, 0]
    planes, hm = c.host()
    assert_inside(out, lse, *attention(c.L, c.lens, c.table, planes, hm, False, c.alpha, INT4, q, None, None))


def test_workspace_is_left_for_other_calls():
    """One workspace, decodes and verifications of other shapes in turn: each time the
    same bits, and the counters zero."""
    big = Case([3000, 10, 700], 4, INT4, bt=16, seed=1)
    small = Case([900], 2, CENTRED, True, seed=2)
    ws = lynx.workspace(big.L, 3, 16, 8, 3000, tree=False)
    a, b = big.queries(16, 1, 0)[0].cuda(), small.queries(8, 4, 0)[0].cuda()
    first = big.call(a), small.call(b)
    for _ in range(3):
        for c, q, want in ((big, a, first[0]), (small, b, first[1])):
            got = c.call(q, ws=ws)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            assert not ws[:lynx.ATTN_COUNTER_BYTES].any()


def test_streams_and_graph():
    """Two streams at once, and a captured call replayed among eager ones on new
    queries and lengths."""
    c = Case([2500, 33, 1200], 4, INT4, bt=32, seed=3)
    qs = [c.queries(16, 1, 0, seed=s)[0].cuda() for s in (11, 12, 13)]
    want = [c.call(q) for q in qs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    wss = [lynx.workspace(c.L, 3, 16, 1, 2500, tree=False) for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            got.append(c.call(qs[i % 3], ws=wss[i % 2]))
    torch.cuda.synchronize()
    for i, (o, l) in enumerate(got):
        assert torch.equal(o, want[i % 3][0]) and torch.equal(l, want[i % 3][1])
    q, (out, lse) = qs[0].clone(), c.call(qs[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call(q, ws=wss[0], out=out, lse=lse)
    for i in (1, 0, 2, 1):
        q.copy_(qs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])
        assert torch.equal(c.call(qs[2])[0], want[2][0])
    lens = c.dev_lens.clone()
    c.dev_lens.copy_(torch.tensor([70, 0, 1], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    again = c.call(q, most=2500)
    assert torch.equal(out, again[0]) and (out[1] == 0).all()
    c.dev_lens.copy_(lens)


@pytest.mark.parametrize("bt", [16, 40])
def test_blocks_past_4_gib_of_a_pool(bt):
    T, Hkv = 200, 2
    per = -(-T // bt)
    blocks = (1 << 32) // (64 * Hkv * bt) + 4 * per  # rows of 64 bytes
    small = Case([T], Hkv, INT4, bt=bt, seed=21)
    q, _, _ = small.queries(8, 1, 0)
    want, _ = small.call(q.cuda())
    ids = blocks - 1 - 3 * torch.arange(per)
    for i in range(2):
        big = torch.zeros(blocks, Hkv * bt * 64, dtype=torch.uint8, device="cuda")
        big[ids.cuda()] = small.planes[i].view(-1, Hkv * bt * 64)[small.table[0].long().cuda()]
        small.planes = (big.view(-1), small.planes[1]) if i == 0 else (small.planes[0], big.view(-1))
    small.L.num_blocks = blocks
    small.dev_table = ids.to(torch.int32).view(1, -1).cuda()
    got, _ = small.call(q.cuda())
    assert torch.equal(got, want)
