"""Captured graphs whose calls take the library's workspace: each goes on
using the buffer that it was captured with, whatever later calls on the stream
need.  Replays are compared with the same calls run eagerly, bit for bit."""
import numpy as np
import pytest

from paper_2607_06763_amd import workloads as W
from tests.attn_ref import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_06763_amd import gdn_attn as A
    from paper_2607_06763_amd import gdn_tree as G
    G.lib()
    return A


def bits(t):
    import torch
    return t.view(torch.int16 if t.element_size() == 2 else torch.int32)


def replay_all(graphs, side):
    """graphs: (graph, inputs' change, eager call, output).  Every graph is replayed after all are there, in both
    orders, with new inputs, eager work on the capture stream and synchronisations between."""
    import torch
    for r in range(3):
        for graph, change, eager, out in graphs if r % 2 else graphs[::-1]:
            change()
            out.fill_(float("nan"))
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                want = eager()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.isfinite(want).all() and torch.equal(bits(out), bits(want))


def capture(call, side):
    """The call run once on the stream and then captured there."""
    import torch
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    torch.cuda.synchronize()
    return graph


def test_attention_graphs_in_rising_order(A):
    """One graph per tree size, as a serving program makes them: a token, a small tree, a large one, a batch."""
    import torch
    side = torch.cuda.Stream()
    graphs = []
    for seed, T, ctx in ((1, 1, [700]), (2, 12, [300, 64]), (3, 128, [900, 200]), (4, 128, [500] * 6)):
        print(f"[gpu] capture attend T={T} B={len(ctx)}", flush=True)
        c = Case(700 + seed, T, ctx, 16, 4, 128, 64, "bf16", parent=None if T == 1 else "any")
        c.append_slots()
        g, d = c.device(), c.dims()
        out = torch.empty_like(g["q"])

        def call(o, d=d, g=g):
            A.attend(d, g["q"], g["kc"], g["vc"], g["table"], g["ctx"], o, meta=g["meta"])
            return o
        change = lambda g=g: g["q"].copy_(torch.randn_like(g["q"], dtype=torch.float32).to(g["q"].dtype))
        graph = capture(lambda: call(out), side)
        graphs.append((graph, change, lambda call=call, out=out: call(torch.empty_like(out)), out))
    replay_all(graphs, side)


def test_verification_graphs_in_rising_order(A):
    """The same above 128 slots, where verify takes a workspace, and for the chunked form."""
    import torch
    from paper_2607_06763_amd import gdn_tree as G
    side = torch.cuda.Stream()
    graphs = []
    for T, chunked in ((140, False), (60, True), (512, False), (300, True)):
        print(f"[gpu] capture verify T={T} chunked={chunked}", flush=True)
        dt = G.DeviceTree(W.make_random(7300 + T, 2, T, 1, 2, 64, 64, "bf16", shuffle=True))
        dt.prepare()
        out = torch.empty_like(dt.out)

        def call(o, dt=dt, chunked=chunked):
            dt.verify(out=o, chunked=chunked)
            return o
        change = lambda dt=dt: dt.q.copy_(torch.randn_like(dt.q, dtype=torch.float32).to(dt.q.dtype))
        graph = capture(lambda: call(out), side)
        graphs.append((graph, change, lambda call=call, out=out: call(torch.empty_like(out)), out))
    replay_all(graphs, side)
