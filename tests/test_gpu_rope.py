"""Norms and rotation of query and key heads against 64 bits: head layouts, rotated
widths and both pairings, with and without norms and V, fused and separate rows,
far positions, skipped tokens and scattered rows, extreme values, streams, graphs."""
import math

import pytest
import torch

from paper_2607_01831_amd import lynx
from tests.gpu_cases import note

pytestmark = pytest.mark.gpu

EPS = 1e-6


def reference(x, w, positions, inv_freq, pairs, scale):
    """(y, bound) float64 [tokens][heads][128].  fp32: the mean and its root within
    2^-20, each product 2^-24, the angle 2^-22 turns; then half a BF16 step, 2^-8."""
    x = x.double().cpu()
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.double().cpu()
    y, size = x.clone(), x.abs()
    if inv_freq is not None:
        half = len(inv_freq)
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if pairs else (slice(0, half), slice(half, 2 * half))
        angle = positions.double().cpu()[:, None] * inv_freq.double().cpu()
        c, s = angle.cos()[:, None] * scale, angle.sin()[:, None] * scale
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        both = (x[..., a].abs() + x[..., b].abs()) * abs(scale)
        size[..., a] = size[..., b] = both
    return y, 2.0 ** -8 * y.abs() + 2.0 ** -18 * size + 1e-38


def heads(tokens, Hq, Hkv, seed, fused=True):
    g = torch.Generator().manual_seed(seed)
    row = torch.randn(tokens, Hq + 2 * Hkv, 128, generator=g).bfloat16().cuda()
    parts = row[:, :Hq], row[:, Hq:Hq + Hkv], row[:, Hq + Hkv:]
    w = [(1 + 0.3 * torch.randn(128, generator=g)).bfloat16().cuda() for _ in range(2)]
    return (parts if fused else [p.contiguous() for p in parts]), w


def freqs(rotary, base=500000.0):
    return (base ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / rotary)).float().cuda() if rotary else None


def check(tokens, Hq, Hkv, rotary, pairs, norm=(True, True), values=True, fused=True, scale=1.0, positions=None, seed=0):
    (q, k, v), w = heads(tokens, Hq, Hkv, seed + tokens, fused)
    w = [x if n else None for x, n in zip(w, norm)]
    if positions is None:
        positions = torch.randint(0, 131072, (tokens,), generator=torch.Generator().manual_seed(seed))
    positions = positions.to(torch.int32).cuda()
    f = freqs(rotary)
    outs = [torch.full((tokens, h, 128), math.nan, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv)]
    if not values:
        v, outs[2] = None, None
    note(f"rope tokens={tokens} Hq={Hq} Hkv={Hkv} rotary={rotary} pairs={pairs} norm={norm} v={values} fused={fused}")
    lynx.lynx_qk_norm_rope(q, k, v, positions, None, *w, EPS, f, pairs, scale, *outs)
    torch.cuda.synchronize()
    for x, weight, got in ((q, w[0], outs[0]), (k, w[1], outs[1])):
        y, bound = reference(x, weight, positions, f, pairs, scale)
        off = (got.double().cpu() - y).abs()
        assert (off <= bound).all(), f"{(off / bound).max():.2f} of the bound"
    if values:
        assert torch.equal(outs[2], v)


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("rotary", [0, 16, 32, 48, 64, 80, 96, 112, 128])
def test_rotated_widths(rotary, pairs):
    check(5, 3, 2, rotary, pairs)
    check(2050, 4, 1, rotary, pairs, values=False)


@pytest.mark.parametrize("tokens", [1, 2, 3, 63, 2047, 2048, 2049, 2051])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 4), (28, 4), (32, 8), (13, 13)])
def test_tokens_and_heads(tokens, Hq, Hkv):
    check(tokens, Hq, Hkv, 128, tokens % 2 == 1, fused=tokens % 3 != 0)


def test_more_tokens_than_a_grid_axis():
    for tokens in (65535, 65536, 131077):
        check(tokens, 1, 1, 16, False, seed=5)


@pytest.mark.parametrize("norm", [(False, False), (True, False), (False, True)])
def test_without_norms(norm):
    for tokens in (7, 2100):
        check(tokens, 8, 2, 128, False, norm=norm, values=False, scale=1.25)
        check(tokens, 8, 2, 64, True, norm=norm, fused=False, scale=-0.5)


def test_far_positions():
    far = torch.tensor([0, 1, 2 ** 24 + 1, 2 ** 30 + 7, 2 ** 31 - 1, 131071, 10 ** 9])
    for pairs in (False, True):
        check(7, 2, 1, 128, pairs, positions=far)


def test_skipped_tokens_and_rows():
    """Negative positions and rows outside the outputs write nothing; the others go
    to their rows, and rows of no token stay as they were."""
    for tokens in (40, 2300):
        (q, k, v), w = heads(tokens, 4, 2, 3)
        g = torch.Generator().manual_seed(tokens)
        n_rows = tokens + 9
        positions = torch.randint(0, 5000, (tokens,), generator=g, dtype=torch.int32)
        rows = torch.randperm(n_rows, generator=g)[:tokens].to(torch.int32)
        positions[3::7] = -1
        positions[5] = -2 ** 31
        rows[4::9] = -1
        rows[8], rows[12] = n_rows, 2 ** 31 - 1
        f = freqs(128)
        plain = [torch.empty(tokens, h, 128, dtype=torch.bfloat16, device="cuda") for h in (4, 2, 2)]
        lynx.lynx_qk_norm_rope(q, k, v, positions.cuda().clamp(min=0), None, *w, EPS, f, False, 1.0, *plain)
        outs = [torch.full((n_rows, h, 128), 7.5, dtype=torch.bfloat16, device="cuda") for h in (4, 2, 2)]
        lynx.lynx_qk_norm_rope(q, k, v, positions.cuda(), rows.cuda(), *w, EPS, f, False, 1.0, *outs)
        for got, src in zip(outs, plain):
            want = torch.full_like(got, 7.5)
            there = ((positions >= 0) & (rows >= 0) & (rows < n_rows)).nonzero()[:, 0]
            want[rows[there].long().cuda()] = src[there.cuda()]
            assert torch.equal(got, want)


def test_padded_outputs_are_rows_in_order():
    """Outputs of more dims, as attention takes them: [B][n][heads][128]."""
    (q, k, v), w = heads(6, 4, 2, 8)
    rows = torch.tensor([0, 1, 2, 4, 8, 9], dtype=torch.int32).cuda()
    pos = torch.arange(6, dtype=torch.int32).cuda()
    outs = [torch.zeros(3, 4, h, 128, dtype=torch.bfloat16, device="cuda") for h in (4, 2, 2)]
    lynx.lynx_qk_norm_rope(q, k, v, pos, rows, *w, EPS, freqs(128), False, 1.0, *outs)
    assert torch.equal(outs[2].view(12, 2, 128)[rows.long()], v)
    with pytest.raises(ValueError):
        lynx.lynx_qk_norm_rope(q, k, v, pos, rows, *w, EPS, freqs(128), False, 1.0, outs[0], outs[1][:2], outs[2])
    with pytest.raises(lynx.LynxError):
        lynx.lynx_qk_norm_rope(q, k, v, pos, None, *w, EPS, freqs(128), False, 1.0, *(x.view(12, -1, 128)[:5] for x in outs))


def test_large_small_and_zero_heads():
    """Heads whose squares are still finite in fp32, heads below eps, zeros; without a
    norm the largest BF16 passes unrotated dims."""
    x = torch.randn(4, 4, 128, generator=torch.Generator().manual_seed(1))
    x[0] *= 1e17
    x[1] *= 1e-20
    x[2] = 0
    q = x.bfloat16().cuda()
    k = q[:, :1].contiguous()
    pos = torch.tensor([5, 6, 7, 8], dtype=torch.int32).cuda()
    w = torch.ones(128, dtype=torch.bfloat16).cuda()
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    for pairs in (False, True):
        lynx.lynx_qk_norm_rope(q, k, None, pos, None, w, w, EPS, freqs(64), pairs, 1.0, qo, ko, None)
        y, bound = reference(q, w, pos, freqs(64), pairs, 1.0)
        assert ((qo.double().cpu() - y).abs() <= bound).all()
        assert (qo[2] == 0).all()
    q[0, 0, 64:] = 3.3895e38
    q[0, 1, 100] = math.inf
    q[0, 2, 127] = math.nan
    lynx.lynx_qk_norm_rope(q, k, None, pos, None, None, None, 0.0, freqs(64), False, 1.0, qo, ko, None)
    assert torch.equal(qo[:, :, 64:].isnan(), q[:, :, 64:].isnan())
    there = ~q[:, :, 64:].isnan()
    assert torch.equal(qo[:, :, 64:][there], q[:, :, 64:][there])
    assert torch.isfinite(qo[:, :, :64]).all()


def test_streams_and_graph():
    (q, k, v), w = heads(37, 8, 2, 5)
    f = freqs(128)
    q, k, v = (x.contiguous() for x in (q, k, v))
    pos = torch.arange(100, 137, dtype=torch.int32).cuda()
    new = lambda: [torch.zeros_like(x) for x in (q, k, v)]  # noqa: E731
    want, got, outs = new(), new(), new()
    lynx.lynx_qk_norm_rope(q, k, v, pos, None, *w, EPS, f, False, 1.0, *want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    lynx.lynx_qk_norm_rope(q, k, v, pos, None, *w, EPS, f, False, 1.0, *got, stream=s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lynx.lynx_qk_norm_rope(q, k, v, pos, None, *w, EPS, f, False, 1.0, *outs)
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        for a, b, c in zip(want, got, outs):
            assert torch.equal(a, b) and torch.equal(a, c)
        q.neg_()
        pos.add_(11 * i)
        want = new()
        lynx.lynx_qk_norm_rope(q, k, v, pos, None, *w, EPS, f, False, 1.0, *want)
        got = want


def test_rows_past_4_gib():
    tokens, Hq = 3, 2
    (q, k, v), w = heads(tokens, Hq, 1, 2)
    n_rows = (1 << 32) // (Hq * 256) + 5
    big = torch.zeros(n_rows, Hq, 128, dtype=torch.bfloat16, device="cuda")
    small = [torch.zeros(n_rows, 1, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    rows = torch.tensor([n_rows - 1, 0, n_rows - 4], dtype=torch.int32).cuda()
    pos = torch.tensor([9, 8, 7], dtype=torch.int32).cuda()
    lynx.lynx_qk_norm_rope(q, k, v, pos, rows, *w, EPS, freqs(128), True, 1.0, big, *small)
    want = [torch.zeros(tokens, h, 128, dtype=torch.bfloat16, device="cuda") for h in (Hq, 1, 1)]
    lynx.lynx_qk_norm_rope(q, k, v, pos, None, *w, EPS, freqs(128), True, 1.0, *want)
    for a, b in zip((big, *small), want):
        assert torch.equal(a[rows.long()], b)
