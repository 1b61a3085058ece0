"""Calls on a stream of their own while the current stream still has work pending on memory that its
owner has given back: the calls' results and workspaces are not in it."""
import math

import pytest
import torch

from paper_2609_04910_amd import attention as at

pytestmark = pytest.mark.gpu


def pending_writes(sizes):
    """Blocks of the current stream, of every one of `sizes` bytes, given back while the kernels that fill them
    wait behind half a second or so of nothing."""
    torch.cuda.synchronize()
    blocks = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(3)]
    torch.cuda._sleep(200_000_000)
    for b in blocks:
        b.fill_(255)                           # NaN of every type


def sizes_of(results, *workspaces):
    return [t.numel() * t.element_size() for t in results] + [n for n in workspaces if n]


def run(call, *workspaces):
    side = torch.cuda.Stream()
    want = [t.clone() for t in call(None)]
    call(side)
    torch.cuda.synchronize()
    for _ in range(2):
        pending_writes(sizes_of(want, *workspaces))
        got = call(side)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("N", [400, 5000])
def test_attention(N):
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn((2, n, h, 64), generator=gen, device="cuda").bfloat16() for n, h in ((60, 4), (N, 2), (N, 2)))
    g = torch.randn(q.shape, generator=gen, device="cuda").bfloat16()
    out, lse = at.attention_fwd(q, k, v)
    run(lambda st: at.attention_fwd(q, k, v, stream=st), at.attention_fwd_workspace_size(2, 60, N, 4, 2, 64, 64))
    run(lambda st: at.attention_bwd(q, k, v, out, lse, g, stream=st), at.attention_bwd_workspace_size(2, 60, N, 4, 2, 64, 64))


def test_attention_over_pages():
    gen = torch.Generator(device="cuda").manual_seed(2)
    q, k, v = (torch.randn((n, h, 64), generator=gen, device="cuda").half() for n, h in ((6, 4), (3000, 2), (3000, 2)))
    kp, vp = (t.view(30, 100, 2, 64) for t in (k, v))
    table = torch.arange(30, dtype=torch.int32, device="cuda").view(2, 15)
    lens = torch.tensor([1500, 900], dtype=torch.int32, device="cuda")
    run(lambda st: at.attention_paged(q, kp, vp, table, lens, return_lse=True, stream=st),
        at.attention_paged_workspace_size(2, 3, 4, 2, 64, 64, 100, 15))
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = at.attention_paged(q, kp, vp, table[:0], lens[:0], q_offsets=none, return_lse=True)
    assert not out.any() and (lse == -math.inf).all()
    run(lambda st: at.attention_paged(q, kp, vp, table[:0], lens[:0], q_offsets=none, return_lse=True, stream=st))


def test_gauss_sums():
    from paper_2609_04910_amd import gauss_sum as gs
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k, v, g = (torch.randn(s, generator=gen, device="cuda") for s in ((700, 32), (900, 32), (900, 4), (700, 4)))
    q, k, weights = q.half(), k.half(), v[:, :1].contiguous()
    run(lambda st: [gs.gauss_sum_fwd(q, k, v, 0.1, stream=st)], gs.gauss_sum_fwd_workspace_size(700, 900, 32, 4))
    run(lambda st: gs.gauss_sum_bwd(q, k, v, 0.1, g, stream=st), gs.gauss_sum_bwd_workspace_size(700, 900, 32, 4))
    run(lambda st: gs.gauss_sum_fwd_bwd(q, k, v, 0.1, g, stream=st), gs.gauss_sum_fwd_bwd_workspace_size(700, 900, 32, 4))
    run(lambda st: gs.gauss_sum_mmd_flow(k, weights, 0.1, stream=st), gs.gauss_sum_mmd_flow_workspace_size(900, 32))
    batched = [t.expand(3, -1, -1).contiguous() for t in (q, k, v, g)]
    run(lambda st: gs.gauss_sum_fwd_bwd_batched(*batched[:3], 0.1, batched[3], stream=st),
        gs.gauss_sum_fwd_bwd_batched_workspace_size(700, 900, 32, 4, 3))


def test_a_call_on_a_stream_forked_in_a_capture():
    gen = torch.Generator(device="cuda").manual_seed(4)
    q, k, v = (torch.randn((2, n, 2, 64), generator=gen, device="cuda").half() for n in (60, 5000, 5000))
    g = torch.randn(q.shape, generator=gen, device="cuda").half()
    side = torch.cuda.Stream()

    def step(stream):
        out, lse = at.attention_fwd(q, k, v, stream=stream)
        return (out, lse) + at.attention_bwd(q, k, v, out, lse, g, stream=stream)

    want = [t.clone() for t in step(None)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        held = step(side)
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        for t in held:
            t.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b)
        step(None)
        torch.cuda.synchronize()
