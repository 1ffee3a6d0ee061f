"""Acceptance calls that make their workspace themselves, on a stream that is not
the current one: it is cleared before the call, and nobody has it until the call
is done, however far either stream is behind the other."""
import pytest
import torch

from paper_2607_01831_amd import lynx
from tests.gpu_cases import note

pytestmark = pytest.mark.gpu

B, N, V = 4, 24, 50257
SPIN = 20_000_000  # cycles


def call_of(kind):
    """(call(stream, workspace), outputs, the workspace's bytes)"""
    g = torch.Generator().manual_seed(3)
    ints = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")  # noqa: E731
    scores = torch.randn(B, N + 1, V, generator=g).cuda()
    tokens, uniforms = scores[:, :-1].argmax(-1).int(), torch.rand(B, N + 1, generator=g).cuda()
    parents = (torch.arange(N, dtype=torch.int32) - 1).repeat(B, 1).cuda()
    probs, drafts = scores.softmax(-1), torch.randn(B, N, V, generator=g).softmax(-1).cuda()
    out = [ints(B), ints(B), ints(B, N)]
    accepted, following, path = out
    f, args, size = {
        "greedy": (lynx.lynx_spec_accept_greedy, (scores, tokens, accepted, following), lynx.lynx_spec_accept_workspace_bytes),
        "sample": (lynx.lynx_spec_accept_sample, (probs, drafts, tokens, uniforms, accepted, following),
                   lynx.lynx_spec_accept_workspace_bytes),
        "tree greedy": (lynx.lynx_spec_accept_tree_greedy, (scores, tokens, parents, accepted, path, following),
                        lynx.lynx_spec_tree_workspace_bytes),
        "tree sample": (lynx.lynx_spec_accept_tree_sample, (probs, tokens, parents, uniforms, accepted, path, following),
                        lynx.lynx_spec_tree_workspace_bytes),
    }[kind]
    return (lambda stream, ws=None: f(*args, ws, stream=stream)), out, size(B, N, V)


@pytest.mark.parametrize("behind", ["current", "side"])
@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("kind", ["greedy", "sample", "tree greedy", "tree sample"])
def test_a_workspace_of_the_calls_own(kind, handle, behind):
    call, out, nbytes = call_of(kind)
    call(None, torch.zeros(nbytes, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    want = [x.clone() for x in out]
    side = torch.cuda.Stream()
    for x in out:
        x.fill_(-7)
    del x
    torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")  # (what the allocator gives next)
    torch.cuda.synchronize()
    note(f"{kind} handle={handle} behind={behind}")
    with torch.cuda.stream(torch.cuda.current_stream() if behind == "current" else side):
        torch.cuda._sleep(SPIN)
    call(side.cuda_stream if handle else side)
    torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")  # another's, while the call may not be done
    side.synchronize()
    got = [x.clone() for x in out]
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)


def test_the_default_stream_by_its_handle():
    call, out, nbytes = call_of("tree greedy")
    call(None)
    torch.cuda.synchronize()
    want = [x.clone() for x in out]
    for x in out:
        x.fill_(-7)
    note("default stream")
    call(0)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(out, want))
