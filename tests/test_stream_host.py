"""A call's stream is one of the device that its tensors are on: the current one."""
import pytest
import torch

from paper_2607_01831_amd import lynx


class Stream:
    device_index, cuda_stream = 3, 0x5000


@pytest.fixture
def current(monkeypatch):
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    return lambda dev: monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: dev, raising=False)


def test_a_stream_of_another_device_is_refused(current):
    current(0)
    empty = lynx.Meta(None, None, None, None)
    L = lynx.Layout(num_kv_heads=1, block_tokens=16, max_blocks_per_seq=1, num_blocks=1, max_tokens=16)
    x = torch.zeros(1, 1, 1, 128)
    for call in (lambda s: lynx.lynx_attn_verify_tree(L, 1, 1, 1, 16, *[None] * 4, empty, *[None] * 5, stream=s),
                 lambda s: lynx.lynx_spec_accept_tree_greedy(x, *[None] * 5, stream=s),
                 lambda s: lynx.lynx_spec_accept_tree_sample(x, *[None] * 6, stream=s),
                 lambda s: lynx.lynx_kv_append(L, 1, 1, None, None, None, None, x, x, None, *[None] * 6, empty, stream=s),
                 lambda s: lynx.lynx_kv_append_begin(L, 1, None, None, None, empty, None, stream=s),
                 lambda s: lynx.lynx_kv_dequant(L, 1, 1, *[None] * 5, empty, None, None, stream=s)):
        with pytest.raises(ValueError, match="stream is one of device 3"):
            call(Stream())


def test_a_stream_of_the_current_device(current):
    current(3)
    assert lynx._here(Stream()) == (3, 0x5000)
    assert lynx._here(0x7000) == (3, 0x7000)  # (a handle does not say whose it is)
