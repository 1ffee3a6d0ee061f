"""The blocks of a step at the ends of what the calls allow."""
import pytest
import torch

from paper_2607_01831_amd import lynx
from tests.gpu_cases import note

pytestmark = pytest.mark.gpu


def test_release_of_nearly_2_31_blocks():
    """65535 sequences of 32768 blocks of a token, all given back: the workgroups'
    last steps go past 2^31."""
    B, per = 65535, 32768
    total = B * per
    assert 2 ** 31 - 65536 < total < 2 ** 31  # (64 workgroups of 1024 threads step by 65536)
    L = lynx.Layout(num_kv_heads=1, block_tokens=1, max_blocks_per_seq=per, num_blocks=2 ** 31 - 1, max_tokens=per)
    table = torch.arange(total, dtype=torch.int32, device="cuda").view(B, per)
    stack = torch.full((L.num_blocks,), -9, dtype=torch.int32, device="cuda")
    state = torch.zeros(2, dtype=torch.int32, device="cuda")
    lens, keep = torch.full((B,), per, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    note(f"blocks_release B={B} bt=1 blocks={total}")
    lynx.lynx_blocks_release(L, B, lens, keep, table, stack, state)
    assert state.tolist() == [total, 0]
    assert (table == -1).all()
    # the first sequence's first block on top
    assert torch.equal(stack[:total], torch.arange(total - 1, -1, -1, dtype=torch.int32, device="cuda"))
    assert (stack[total:] == -9).all()
