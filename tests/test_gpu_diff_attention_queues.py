"""Differential attention with more items than workgroups, so that every kernel draws tickets: calls that overlap on two streams, graphs that
are replayed beside each other and beside eager calls, and the counters behind them."""
import ctypes as C
import os

import numpy as np
import pytest

from gpu_util import say

LENS = [700, 130, 257, 512, 1, 0, 333, 900, 64] * 3
H = 24


def items(tile):
    return H * sum(-(-n // tile) for n in LENS)


def counters():
    """The library's work-queue counters of this device, as they are now."""
    import torch
    import paper_2508_06001_amd as K
    hip = C.CDLL("libamdhip64.so.7", mode=os.RTLD_NOLOAD | C.RTLD_GLOBAL)      # the runtime that is loaded, never a second one
    hip.hipMemcpy.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int]
    n = C.c_int()
    at = K.lib.knap_fwd_queue_counters(C.byref(n))
    host = np.full((n.value,), -1, dtype=np.int32)
    torch.cuda.synchronize()
    assert hip.hipMemcpy(host.ctypes.data, at, 4 * n.value, 2) == 0
    return host


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_draws_on_two_streams_and_in_graphs_beside_each_other(d, causal):
    import torch
    import paper_2508_06001_amd as K
    assert items(128) > 3 * 256 and items(256) > 256      # workgroups: at most three a CU at 128 rows an item, one at 256
    say(f"[gpu] diff queues d={d} causal={causal} items={items(128)} {items(256)}")
    cu = np.concatenate([[0], np.cumsum(LENS)]).astype(np.int32)
    T = int(cu[-1])
    g = torch.Generator(device="cuda").manual_seed(31 + d)
    x = [[torch.randn((T, H, d), generator=g, device="cuda").bfloat16() for _ in range(4)] for _ in range(2)]
    lam = torch.rand((H,), generator=g, device="cuda")
    new = lambda: K.VarlenDiffAttention(cu, H, d, 0.125, lam, causal=causal)  # noqa: E731

    def step(a, of):
        q, k, v, do = of
        a.forward(q, k, v)
        a.backward(q, k, v, do)

    def results(a):
        return [a.out, a.out2, a.lse, a.dq, a.dk, a.dv, a.dlam]

    def blank(a):
        for t in results(a):
            t.fill_(float("nan"))

    alone = [new() for _ in range(2)]
    for a, of in zip(alone, x):
        step(a, of)
    want = [[t.clone() for t in results(a)] for a in alone]
    torch.cuda.synchronize()
    assert all(bool(torch.isfinite(t).all()) for w in want for t in w)
    streams, twins = [torch.cuda.Stream() for _ in range(2)], [new() for _ in range(2)]
    for turn in range(4):
        for a in twins:
            blank(a)
        torch.cuda.synchronize()
        for s, a, of in zip(streams, twins, x):
            with torch.cuda.stream(s):
                step(a, of)
        torch.cuda.synchronize()
        for a, w in zip(twins, want):
            assert all(torch.equal(t, y) for t, y in zip(results(a), w)), turn
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph, s, a, of in zip(graphs, streams, twins, x):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=s):
            step(a, of)
    torch.cuda.synchronize()
    for turn in range(4):
        for a in twins + alone:
            blank(a)
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        step(alone[0], x[0])                 # an eager call beside them
        torch.cuda.synchronize()
        for a, w in ((twins[0], want[0]), (twins[1], want[1]), (alone[0], want[0])):
            assert all(torch.equal(t, y) for t, y in zip(results(a), w)), turn
    assert not counters().any()              # every launch left its set at zero
