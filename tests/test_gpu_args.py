"""The binding's test of a tensor argument: the C++ form gives and refuses what
the Python form does."""
import pytest
import torch

from paper_2607_01831_amd import lynx

pytestmark = pytest.mark.gpu

BF16, I32 = torch.bfloat16, torch.int32


def both(*args):
    out = []
    for f in (lynx._args.typed, lynx._typed_form):
        try:
            out.append(f("call", "x", *args))
        except Exception as e:  # noqa: BLE001
            out.append((type(e), str(e)))
    return out


def test_what_passes():
    x = torch.zeros(6, 4, dtype=BF16, device="cuda")
    assert lynx._typed is lynx._args.typed
    for t, size in ((x, 48), (x, 0), (x, 1), (x[2:], 32), (x[:, :1].contiguous(), 12), (x[:0], 0)):
        assert both(t, size, BF16, 0) == [t.data_ptr()] * 2
    assert both(None, 5, BF16, 0) == [None] * 2
    assert both(1234, 5, BF16, 0) == [1234] * 2


@pytest.mark.parametrize("what", ["short", "type", "device", "other device", "strides", "no tensor", "meta", "huge"])
def test_what_is_refused(what):
    x = torch.zeros(6, 4, dtype=BF16, device="cuda")
    args = {"short": (x, 50, BF16, 0), "type": (x, 8, I32, 0), "device": (x.cpu(), 8, BF16, 0),
            "other device": (x, 8, BF16, 1), "strides": (x[:, ::2], 8, BF16, 0), "no tensor": ([1, 2], 8, BF16, 0),
            "meta": (x.to("meta"), 8, BF16, 0), "huge": (x, 2 ** 70, BF16, 0)}[what]
    fast, plain = both(*args)
    assert fast == plain and isinstance(plain, tuple)
