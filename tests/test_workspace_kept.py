"""Buffers larger than a replay needs: one that a device call has used, and a graph may therefore name, is kept when it is outgrown."""
import contextlib

import numpy as np
import pytest


class _Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


def has(buffers, t):
    return any(x is t for x in buffers)


def test_what_is_kept(monkeypatch):
    import paper_2608_30310_b200 as gdn
    from paper_2608_30310_b200 import _binding as B
    monkeypatch.setattr(B, "_on_stream", lambda s: contextlib.nullcontext())
    ws, a, b = gdn.Workspace(device="cpu"), _Stream(0), _Stream(7)
    staging = ws.reserve(30 << 20, a)                                      # a call on host memory
    used = ws.reserve(30 << 20, b)
    assert ws.reserve(1 << 10, b, device_call=True) is used                # a device call takes what is there
    assert ws.reserve(40 << 20, a) is not staging and ws.reserve(40 << 20, b) is not used
    assert has(ws.outgrown, used) and not has(ws.outgrown, staging)
    large = ws.reserve(50 << 20, b, device_call=True)                      # one that needs so much itself
    ws.reserve(60 << 20, b)
    assert has(ws.outgrown, large)
    last = ws.by_stream[7]
    ws.reserve(70 << 20, b)                                                # (the mark was the other buffer's)
    assert not has(ws.outgrown, last)
    ws.buf = None
    assert not ws.kept and not ws.outgrown


@pytest.mark.gpu
@pytest.mark.parametrize("before", [0, 40 << 20])
def test_a_captured_compaction_outlives_the_growth_of_its_workspace(before):
    """1.2 million pages need 14 MB; or a call on host memory has left a larger buffer, which the compaction takes."""
    import torch
    import paper_2608_30310_b200 as gdn
    P = 1200000
    count = np.random.default_rng(1).integers(0, 2, size=P).astype(np.int32)
    live = int((count > 0).sum())
    counts, tables = torch.from_numpy(count).cuda(), torch.full((1, 4), -1, dtype=torch.int32, device="cuda")
    pool = torch.arange(P * 4, dtype=torch.int32, device="cuda").view(P, 4)
    oc, ot, page_map, n = torch.empty_like(counts), torch.empty_like(tables), torch.empty_like(counts), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws, side, graph = gdn.Workspace(), torch.cuda.Stream(), torch.cuda.CUDAGraph()

    def call():
        gdn.gdn_cache_compact([pool], counts, tables, oc, ot, page_map, n, workspace=ws, stream=side)
    torch.cuda.synchronize()
    if before:
        ws.ensure(before, side)
    call()
    call()
    side.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call()
    first = ws.by_stream[side.cuda_stream]
    ws.ensure(100 << 20, side)
    assert has(ws.outgrown, first)
    pool.copy_(torch.arange(P * 4, dtype=torch.int32, device="cuda").view(P, 4))
    page_map.zero_()
    graph.replay()
    torch.cuda.synchronize()
    holes, late = np.flatnonzero(count[:live] == 0), live + np.flatnonzero(count[live:])
    want = np.arange(P)
    want[holes] = late
    assert int(n) == live and torch.equal(pool[:live, 0].cpu().long(), torch.from_numpy(want[:live] * 4))
    to = np.where(count > 0, np.arange(P), -1)
    to[late] = holes
    assert torch.equal(page_map.cpu().long(), torch.from_numpy(to))


@pytest.mark.gpu
def test_a_captured_replay_outlives_the_staging_whose_buffer_it_took():
    import torch
    import oracle
    import paper_2608_30310_b200 as gdn
    from gdn_workloads import make_inputs
    from gpu_utils import assert_parity, to_torch
    inp = make_inputs([300], 2, 4, 128, 128, "bf16", seed=971)
    x = to_torch(inp, "cuda")
    o, st = torch.empty_like(x[2]), torch.empty((1, 4, 128, 128), device="cuda")
    ws, side, graph = gdn.Workspace(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    ws.ensure(40 << 20, side)
    staging = ws.by_stream[side.cuda_stream]
    with torch.cuda.graph(graph, stream=side):
        gdn.gdn_tail_replay(*x, 64, o, st, workspace=ws, stream=side)
        gdn.gdn_tail_replay(*x, 64, o, st, workspace=ws, stream=side)
    ws.ensure(100 << 20, side)
    assert has(ws.outgrown, staging)
    o.zero_()
    st.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert_parity(inp, o.float().cpu().numpy(), st.cpu().numpy(), *oracle.gdn_forward_inputs(inp))
