"""Hierarchical attention with fewer workers than sequences: so many rows that a kv
head's chunks of them take most of the workgroups there are."""
import numpy as np
import pytest

from tests.hier_ref import CENTRED, INT4
from tests.test_gpu_hier_attn import Case

pytestmark = pytest.mark.gpu


# workers: 512 / (rows a kv head / 32 x kv heads)
@pytest.mark.parametrize("B,most,Hkv,G,k,tail,bt,full", [
    (10, 1500, 1, 64, 64, 64, 16, False), (7, 2600, 4, 32, 32, 0, None, True), (64, 130, 1, 32, 64, 0, 16, False),
    (30, 700, 2, 64, 16, 20, 24, True), (9, 1100, 1, 64, 64, 0, 48, False)])
def test_fewer_workers_than_sequences(B, most, Hkv, G, k, tail, bt, full):
    assert B > 512 // (k * G // 32 * Hkv)
    r = np.random.default_rng(B)
    lens = [0 if i % 5 == 2 else int(r.integers(1, most)) for i in range(B)]
    Case(lens, Hkv, CENTRED if full else INT4, full, bt=bt, seed=B).check(Hkv * G, k, tail)

