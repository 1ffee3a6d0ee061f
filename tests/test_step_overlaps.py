"""Arrays of the head norms with rotation that overlap are refused before anything is
launched (no pointer below is dereferenced)."""
import itertools

import pytest

from paper_2607_01831_amd import lynx as E

M = 1 << 20
OUTS = ("q_out", "k_out", "v_out")
N, HQ, HKV, ROTARY, STRIDE = 40, 8, 2, 96, 1536
SIZES = dict(q=((N - 1) * STRIDE + HQ * 128) * 2, k=((N - 1) * STRIDE + HKV * 128) * 2, v=((N - 1) * STRIDE + HKV * 128) * 2,
             positions=4 * N, rows=4 * N, q_weight=256, k_weight=256, inv_freq=2 * ROTARY, q_out=N * HQ * 256, k_out=N * HKV * 256,
             v_out=N * HKV * 256)


@pytest.fixture(scope="module")
def lib():
    if not E.LIBRARY.exists():
        from paper_2607_01831_amd import build
        build.build()
    return E.load()


def call(lib, **at):
    p = {name: M * (i + 1) for i, name in enumerate(SIZES)}
    p.update(at)
    return lib.lynx_qk_norm_rope(N, HQ, HKV, 128, p["q"], STRIDE, p["k"], STRIDE, p["v"], STRIDE, p["positions"], p["rows"], N,
                                 p["q_weight"], p["k_weight"], 1e-6, p["inv_freq"], ROTARY, 0, 1.0, p["q_out"], p["k_out"],
                                 p["v_out"], None)


@pytest.mark.parametrize("out,other", [(a, b) for a, b in itertools.product(OUTS, SIZES) if a != b])
def test_outputs_over_any_other_array(lib, out, other):
    base = 64 * M
    for at in (base, base + SIZES[out] - 16, base - SIZES[other] // 16 * 16 + (0 if SIZES[other] % 16 else 16)):
        assert call(lib, **{out: base, other: at}) == E.LYNX_EINVAL, at
