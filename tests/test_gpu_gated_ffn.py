"""Gated feed-forward block against the oracle in 64 bits, at its bounds (oracle/gated_ffn.py): tokens from one on, sizes around every tile, both
activations, strides, what is not wanted, both directions; captured calls, other streams; and refusals."""
import pytest

from gpu_util import say
from oracle import gated_ffn as G

SIZES = [(1, 8, 8), (1, 64, 128), (2, 72, 40), (3, 768, 2048), (7, 1536, 520), (16, 264, 1000), (17, 512, 512), (31, 136, 72), (32, 1000, 264), (33, 256, 256),
         (64, 64, 64), (65, 200, 328), (100, 2048, 1368), (127, 128, 128), (128, 128, 64), (129, 392, 136), (255, 8, 512), (257, 256, 8), (300, 1032, 776),
         (613, 1000, 2664), (1000, 64, 4096), (2049, 520, 1032), (4173, 768, 2048), (5000, 1536, 264)]


def inputs(T, D, F, seed=0, pad=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed + T + 3 * D + 7 * F)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()  # noqa: E731
    x, dy = new(T, D + pad)[:, pad // 2:pad // 2 + D], new(T, D + pad)[:, :D]
    return x, (new(F, D) / D ** 0.5), (new(F, D) / D ** 0.5), (new(D, F) / F ** 0.5), dy


class Guarded:
    """A contiguous or strided view of NaN between NaN."""

    def __init__(self, rows, cols, pad=0):
        import torch
        self.big = torch.full((rows + 2, cols + pad), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.view = self.big[1:-1, :cols]
        self.cols = cols

    def check(self, name):
        import torch
        assert bool(torch.isnan(self.big[0]).all()) and bool(torch.isnan(self.big[-1]).all()) and bool(torch.isnan(self.big[:, self.cols:]).all()), name
        assert bool(torch.isfinite(self.view).all()), name


def run(T, D, F, gelu, seed=0, pad=0, backward=True):
    import torch
    import paper_2508_06001_amd as K
    say(f"[gpu] ffn T={T} D={D} F={F} gelu={gelu} pad={pad}")
    x, wg, wu, wd, dy = inputs(T, D, F, seed, pad)
    act = K.KNAP_GELU_TANH if gelu else K.KNAP_SILU
    shapes = {"gate": (T, F), "up": (T, F), "h": (T, F), "y": (T, D), "dx": (T, D), "dw_gate": (F, D), "dw_up": (F, D), "dw_down": (D, F)}
    o = {n: Guarded(*s, pad if n in ("y", "dx") else 0) for n, s in shapes.items()}
    v = {n: t.view for n, t in o.items()}
    ws = torch.full((max(256, K.knap_gated_ffn_fwd_workspace_bytes(T, D, F), K.knap_gated_ffn_bwd_workspace_bytes(T, D, F)),), 255, dtype=torch.uint8,
                    device="cuda")
    if not backward:
        K.knap_gated_ffn_fwd(x, wg, wu, wd, act, None, None, v["h"], v["y"], ws)
    else:
        K.knap_gated_ffn_fwd(x, wg, wu, wd, act, v["gate"], v["up"], v["h"], v["y"], ws)
        K.knap_gated_ffn_bwd(x, wg, wu, wd, act, v["gate"], v["up"], v["h"], dy, v["dx"], v["dw_gate"], v["dw_up"], v["dw_down"], ws)
    torch.cuda.synchronize()
    val, off = G.gated_ffn(*(t.double() for t in (x, wg, wu, wd)), gelu, dy.double() if backward else None)
    for n in val if backward else ("h", "y"):
        o[n].check(n)
        far = G.worst_block(v[n], val[n], off[n])
        assert far <= 1.0, (n, far)
    return v


@pytest.mark.gpu
@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("T,D,F", SIZES)
def test_sizes(T, D, F, gelu):
    run(T, D, F, gelu)
    run(T, D, F, gelu, backward=False)


@pytest.mark.gpu
@pytest.mark.parametrize("T", list(range(1, 20)) + [47, 48, 49, 63, 64, 65, 79, 80, 81, 96, 97, 111, 112, 113, 143, 160, 161, 191, 192, 193])
def test_numbers_of_tokens(T):
    run(T, 264, 520, False, backward=T % 4 == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("D,F", [(4104, 4104), (1032, 16400), (16392, 1096), (264, 8), (768, 2048)])
@pytest.mark.parametrize("T", [17, 24, 32, 33, 47, 64, 65])
def test_few_tokens_of_larger_weights(T, D, F):
    run(T, D, F, T % 2 == 0, backward=T in (24, 47))


@pytest.mark.gpu
@pytest.mark.parametrize("T,D,F", [(5, 72, 136), (70, 256, 264), (300, 520, 1032), (3000, 1536, 2056)])
def test_strides(T, D, F):
    run(T, D, F, False, pad=16)


@pytest.mark.gpu
@pytest.mark.parametrize("T,D,F", [(9000, 2048, 5504), (12001, 1544, 4104)])
def test_many_tiles(T, D, F):
    run(T, D, F, T % 2 == 0)


@pytest.mark.gpu
def test_wanted_or_not_every_gradient_has_the_same_bits_and_again():
    import torch
    import paper_2508_06001_amd as K
    for T, D, F in ((33, 256, 264), (613, 1000, 2664)):
        x, wg, wu, wd, dy = inputs(T, D, F)
        f = K.GatedFeedForward(T, D, F, wg, wu, wd)
        y = f.forward(x).clone()
        whole = [t.clone() for t in f.backward(x, dy)]
        f.workspace.fill_(255)
        assert torch.equal(f.forward(x), y) and all(torch.equal(a, b) for a, b in zip(whole, f.backward(x, dy)))
        inference = K.GatedFeedForward(T, D, F, wg, wu, wd, train=False)
        assert torch.equal(inference.forward(x), y)
        new = [torch.full_like(t, float("nan")) for t in whole]
        back = lambda *w: K.knap_gated_ffn_bwd(x, wg, wu, wd, K.KNAP_SILU, f.gate, f.up, f.h, dy, *w, f.workspace)  # noqa: E731
        val, off = G.gated_ffn(*(t.double() for t in (x, wg, wu, wd)), False, dy.double())
        back(new[0], None, None, None)
        assert torch.equal(new[0], whole[0])
        for wants in ((1,), (2,), (3,), (1, 2), (2, 3), (1, 3)):       # parts of sums may be cut elsewhere: at the bounds
            back(None, *(new[i] if i in wants else None for i in (1, 2, 3)))
            for i in wants:
                n = ("dx", "dw_gate", "dw_up", "dw_down")[i]
                assert G.worst_block(new[i], val[n], off[n]) <= 1.0, (n, wants)
                new[i].fill_(float("nan"))


@pytest.mark.gpu
def test_no_tokens():
    import torch
    import paper_2508_06001_amd as K
    _, wg, wu, wd, _ = inputs(1, 64, 72)
    f = K.GatedFeedForward(0, 64, 72, wg, wu, wd)
    x = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    for t in (f.dw_gate, f.dw_up, f.dw_down):
        t.fill_(3.0)
    f.forward(x)
    f.backward(x, x)
    torch.cuda.synchronize()
    assert not any(bool(t.any()) for t in (f.dw_gate, f.dw_up, f.dw_down))


@pytest.mark.gpu
@pytest.mark.parametrize("gelu", [False, True])
def test_values_far_from_zero_and_not_finite(gelu):
    """a of up to 3e38 and far below zero: act is a, or zero, and so are its slopes; a bad row stays in its row."""
    import torch
    import paper_2508_06001_amd as K
    act = K.KNAP_GELU_TANH if gelu else K.KNAP_SILU
    D = F = 64
    eye = torch.eye(64, device="cuda").bfloat16()
    x = torch.randn((40, D), device="cuda").bfloat16()
    big = torch.tensor([1e30, -1e30, 1e4, -1e4, 200.0, -200.0, 30.0, -30.0, 17.0, -17.0, 0.0, -0.0], device="cuda").bfloat16()
    x[3, :12] = big
    x[20, 5] = float("nan")
    x[30, 9] = float("inf")
    dy = torch.ones_like(x)
    half = (0.5 * eye.float()).bfloat16()
    small = (1e-30 * eye.float()).bfloat16()
    f = K.GatedFeedForward(40, D, F, eye, small, half, act)       # b = 1e-30 x: h of 1e30 is 1e30
    y = f.forward(x)
    dx = f.backward(x, dy)[0]
    torch.cuda.synchronize()
    rows = torch.ones((40,), dtype=torch.bool, device="cuda")
    rows[[20, 30]] = False
    for t in (y, dx):
        assert bool(torch.isfinite(t[rows]).all()) and not bool(torch.isfinite(t[~rows]).all())
    val, off = G.gated_ffn(x[rows].double(), eye.double(), small.double(), half.double(), gelu, dy[rows].double())
    for n, t in (("y", y), ("dx", dx)):       # diagonal weights: every element by itself
        assert bool(((t[rows].double() - val[n]).abs() <= 2 * off[n] + 1e-38).all()), n


@pytest.mark.gpu
def test_captured_calls_follow_their_inputs():
    import torch
    import paper_2508_06001_amd as K
    for T, D, F in ((3, 512, 1032), (700, 264, 1096)):
        x, wg, wu, wd, dy = inputs(T, D, F)
        a, b = (K.GatedFeedForward(T, D, F, wg, wu, wd, K.KNAP_GELU_TANH) for _ in range(2))
        results = lambda f: [f.y, f.h, f.gate, f.up, f.dx, f.dw_gate, f.dw_up, f.dw_down]  # noqa: E731
        a.forward(x)
        a.backward(x, dy)
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=stream):
            b.forward(x)
            b.backward(x, dy)
        for turn in range(4):
            x.normal_()
            dy.normal_()
            wd.mul_(-0.5)
            graph.replay()
            a.workspace.fill_(255)
            a.forward(x)
            a.backward(x, dy)
            torch.cuda.synchronize()
            assert all(torch.equal(s, t) for s, t in zip(results(a), results(b))), turn


@pytest.mark.gpu
def test_two_streams_at_once():
    import torch
    import paper_2508_06001_amd as K
    T, D, F = 900, 520, 1032
    x, wg, wu, wd, dy = inputs(T, D, F)
    one = K.GatedFeedForward(T, D, F, wg, wu, wd)
    want = [one.forward(x).clone()] + [t.clone() for t in one.backward(x, dy)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    blocks = [K.GatedFeedForward(T, D, F, wg, wu, wd) for _ in range(2)]
    for _ in range(5):
        for s, f in zip(streams, blocks):
            f.forward(x, stream=s)
            f.backward(x, dy, stream=s)
    torch.cuda.synchronize()
    for f in blocks:
        assert all(torch.equal(a, b) for a, b in zip(want, [f.y, f.dx, f.dw_gate, f.dw_up, f.dw_down]))


FWD = dict(x=1 << 12, xs=64, tokens=4, width=64, hidden=72, wg=2 << 12, wu=3 << 12, wd=4 << 12, act=0, gate=5 << 12, up=6 << 12, h=7 << 12, y=8 << 12, ys=64,
           ws=9 << 12, nbytes=1 << 30)
BWD = dict(x=1 << 12, xs=64, tokens=4, width=64, hidden=72, wg=2 << 12, wu=3 << 12, wd=4 << 12, act=0, gate=5 << 12, up=6 << 12, h=7 << 12, dy=8 << 12, dys=64,
           dx=10 << 12, dxs=64, dwg=11 << 12, dwu=12 << 12, dwd=13 << 12, ws=9 << 12, nbytes=1 << 30)


def test_bad_arguments_are_refused_without_touching_a_gpu():
    import paper_2508_06001_amd as K
    bad = K.KNAP_ERR_INVALID_ARG
    fwd = lambda **kw: K.lib.knap_gated_ffn_fwd(*{**FWD, **kw}.values(), 0)  # noqa: E731
    bwd = lambda **kw: K.lib.knap_gated_ffn_bwd(*{**BWD, **kw}.values(), 0)  # noqa: E731
    assert fwd(tokens=0, x=0, y=0, h=0) == K.KNAP_OK and bwd(tokens=0, x=0, dy=0, dx=0, dwg=0, dwu=0, dwd=0, ws=0) == K.KNAP_OK
    for wrong in (dict(tokens=-1), dict(tokens=(1 << 26) + 1), dict(width=0), dict(width=60), dict(width=K.KNAP_FFN_MAX_WIDTH + 8, xs=1 << 17), dict(hidden=4),
                  dict(hidden=70), dict(hidden=K.KNAP_FFN_MAX_WIDTH + 8), dict(act=2), dict(act=-1), dict(wg=0), dict(wu=8), dict(wd=(4 << 12) + 2), dict(x=0),
                  dict(x=8), dict(xs=63), dict(xs=68), dict(xs=56), dict(xs=(1 << 20) + 8), dict(h=0), dict(gate=0), dict(up=0), dict(h=(7 << 12) + 8),
                  dict(ws=(9 << 12) + 128)):
        assert fwd(**wrong) == bad, wrong
        assert bwd(**wrong) == bad, wrong
    for wrong in (dict(y=0), dict(y=4), dict(ys=8), dict(y=1 << 12), dict(y=7 << 12), dict(h=1 << 12), dict(gate=6 << 12), dict(gate=7 << 12), dict(up=8 << 12)):
        assert fwd(**wrong) == bad, wrong
    for wrong in (dict(dy=0), dict(dy=8), dict(dys=8), dict(dx=8), dict(dxs=65), dict(dx=1 << 12), dict(dx=8 << 12), dict(dx=11 << 12), dict(dwg=12 << 12),
                  dict(dwu=3 << 12), dict(dwd=7 << 12), dict(dwd=9 << 12), dict(dwg=2), dict(ws=0)):
        assert bwd(**wrong) == bad, wrong
    need = K.knap_gated_ffn_bwd_workspace_bytes(4, 64, 72)
    assert need >= 2 * 4 * 72 * 2 and bwd(nbytes=need - 1) == K.KNAP_ERR_WORKSPACE_TOO_SMALL
    T, D, F = 613, 1000, 2664
    need = K.knap_gated_ffn_fwd_workspace_bytes(T, D, F)
    big = dict(tokens=T, width=D, hidden=F, xs=D, ys=D)
    if need:
        assert fwd(**big, ws=0) == bad and fwd(**big, nbytes=need - 1) == K.KNAP_ERR_WORKSPACE_TOO_SMALL
    for args in ((0, 64, 64), (-1, 64, 64), (4, 0, 64), (4, 64, -8), ((1 << 26) + 1, 64, 64)):
        assert K.knap_gated_ffn_fwd_workspace_bytes(*args) == K.knap_gated_ffn_bwd_workspace_bytes(*args) == 0


@pytest.mark.gpu
def test_the_binding_refuses_what_the_library_cannot_see():
    import torch
    import paper_2508_06001_amd as K
    x, wg, wu, wd, dy = inputs(4, 64, 72)
    f = K.GatedFeedForward(4, 64, 72, wg, wu, wd)
    good = dict(x=x, w_gate=wg, w_up=wu, w_down=wd, act=K.KNAP_SILU, gate=f.gate, up=f.up, h=f.h, y=f.y, workspace=f.workspace)
    K.knap_gated_ffn_fwd(**good)
    for wrong in (dict(x=x.float()), dict(x=x[:, :56]), dict(x=x.t().contiguous().t()), dict(y=f.y[:3]), dict(y=f.y.float()), dict(w_up=wu[:64]), dict(w_down=wd.t()),
                  dict(w_gate=wg.float()), dict(h=f.h[:3]), dict(gate=f.gate[:, :64]), dict(up=None), dict(workspace=f.workspace[:64]), dict(x=x.cpu()), dict(x=x[0])):
        if "workspace" in wrong and not K.knap_gated_ffn_fwd_workspace_bytes(4, 64, 72):
            continue
        with pytest.raises(K.KnapError):
            K.knap_gated_ffn_fwd(**{**good, **wrong})
    good = dict(x=x, w_gate=wg, w_up=wu, w_down=wd, act=K.KNAP_SILU, gate=f.gate, up=f.up, h=f.h, dy=dy, dx=f.dx, dw_gate=f.dw_gate, dw_up=f.dw_up,
                dw_down=f.dw_down, workspace=f.workspace)
    K.knap_gated_ffn_bwd(**good)
    for wrong in (dict(dx=f.dx[:3]), dict(dx=f.dx.float()), dict(dw_gate=f.dw_gate.float()), dict(dw_up=f.dw_up[:64]), dict(dw_down=f.dw_down.t()), dict(dy=dy[:, :56]),
                  dict(workspace=None), dict(gate=f.gate.float())):
        with pytest.raises(K.KnapError):
            K.knap_gated_ffn_bwd(**{**good, **wrong})
