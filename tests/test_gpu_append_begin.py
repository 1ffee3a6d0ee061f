"""lynx_kv_append_begin over a table with block ids outside the pool: every row of the
open group and the one before it is written, so that what the ring held before has
no part in the groups that appends make of them."""
import numpy as np
import pytest
import torch

from paper_2607_01831_amd import lynx
from tests.gpu_cases import build_cache, note, random_kv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [-1, 2 ** 31 - 1])
@pytest.mark.parametrize("Hkv", [1, 2, 8])
def test_rows_outside_the_pool_are_zero(Hkv, bad):
    T, bt = 300, 16
    c = build_cache(*[[x] for x in random_kv(T, Hkv, seed=3)], Hkv, bt=bt, max_tokens=320, with_oracle=False)
    rings = []
    clean = c.table.clone()
    for fill in (float("nan"), 1e30):
        ring = torch.full((1, lynx.OPEN_ROWS, Hkv, 128), fill, dtype=torch.bfloat16, device="cuda")
        c.table = clean.clone()
        c.table[0, [9, 18]] = bad  # tokens 144.. and 288.. of the groups from 128 and 256 on
        note(f"append_begin Hkv={Hkv} bad={bad}")
        lynx.lynx_kv_append_begin(c.L, 1, c.lens_dev(), c.table_dev(), c.pool.k_codes, c.pool.meta, ring)
        torch.cuda.synchronize()
        rings.append(ring.float().cpu().numpy()[0])
    good = torch.full((1, lynx.OPEN_ROWS, Hkv, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    c.table = clean
    lynx.lynx_kv_append_begin(c.L, 1, c.lens_dev(), c.table_dev(), c.pool.k_codes, c.pool.meta, good)
    good = good.float().cpu().numpy()[0]
    for t in range(128, T):
        for ring in rings:
            assert np.array_equal(ring[t % 256], good[t % 256] * (t // bt not in (9, 18))), t
    for t in range(T, 384):  # not written
        assert np.isnan(rings[0][t % 256]).all()
