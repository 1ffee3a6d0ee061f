"""Head norms with rotation on arrays that stand next to one another in one
allocation: touching is no overlap."""
import pytest
import torch

from paper_2607_01831_amd import lynx
from tests.gpu_cases import note
from tests.test_gpu_rope import EPS, freqs, heads

pytestmark = pytest.mark.gpu


def test_arrays_next_to_one_another():
    N, Hq, H, rotary = 12, 4, 2, 96
    (q, k, v), w = heads(N, Hq, H, seed=3)
    positions = torch.arange(100, 100 + N, dtype=torch.int32, device="cuda")
    rows = torch.randperm(N, generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()
    f = freqs(rotary)
    outs = [torch.zeros(N, h, 128, dtype=torch.bfloat16, device="cuda") for h in (Hq, H, H)]
    note("rope, separate arrays")
    lynx.lynx_qk_norm_rope(q, k, v, positions, rows, *w, EPS, f, False, 1.0, *outs)
    # outputs in front of and behind every input
    order = [positions, outs[0], torch.cat([q, k, v], 1), outs[1], rows, w[0], outs[2], w[1], f]
    buffer = torch.zeros(sum(x.nbytes for x in order), dtype=torch.uint8, device="cuda")
    at, new = 0, []
    for x in order:
        new.append(buffer[at:at + x.nbytes].view(x.dtype).view(x.shape))
        new[-1].copy_(torch.zeros_like(x) if any(x is o for o in outs) else x)
        at += x.nbytes
    p, q_out, row, k_out, r, qw, v_out, kw, inv = new
    note("rope, one allocation")
    lynx.lynx_qk_norm_rope(row[:, :Hq], row[:, Hq:Hq + H], row[:, Hq + H:], p, r, qw, kw, EPS, inv, False, 1.0, q_out, k_out, v_out)
    for got, want in zip((q_out, k_out, v_out), outs):
        assert torch.equal(got, want) and want.any()
    over = row.view(-1)[-N * H * 128:].view(N, H, 128)  # the last tokens' heads
    with pytest.raises(lynx.LynxError):
        lynx.lynx_qk_norm_rope(row[:, :Hq], row[:, Hq:Hq + H], row[:, Hq + H:], p, r, qw, kw, EPS, inv, False, 1.0, q_out, k_out, over)
    with pytest.raises(lynx.LynxError):  # weights that stand in an output
        lynx.lynx_qk_norm_rope(q, k, v, p, r, k_out.view(-1)[:128], kw, EPS, inv, False, 1.0, q_out, k_out, v_out)
