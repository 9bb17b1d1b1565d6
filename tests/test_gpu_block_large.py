"""Residual norm and gated feed-forward on tensors of more than 2^32 bytes: what lies behind that offset against the oracles in 64 bits, everything
else being zeros.  Bars as in the operators' own tests."""
import numpy as np
import pytest

from gpu_util import say
from oracle import gated_ffn as G
from oracle import residual_norm as R

EPS, ALPHA, LAST = float(np.float32(1e-5)), 0.75, 501
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,width,name", [(1_060_001, 2048, "bf16"), (1_080_001, 1003, "fp32")])
def test_residual_norm(rows, width, name):
    import torch
    import paper_2508_06001_amd as K
    say(f"[gpu] large residual norm {rows} x {width} {name}")
    dtype = torch.bfloat16 if name == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(width)
    x, f, dx_out, dy = (torch.zeros((rows, width), dtype=dtype, device="cuda") for _ in range(4))
    for t in (x, f, dx_out, dy):
        assert t.numel() * t.element_size() > 2 ** 32
        t[-LAST:] = torch.randn((LAST, width), generator=g, device="cuda").to(dtype)
    gate, scale, shift = (0.5 * torch.randn((2, width), generator=g, device="cuda") for _ in range(3))
    shift[0] = 0.0
    weight, post_weight = (1 + 0.5 * torch.randn((width,), generator=g, device="cuda") for _ in range(2))
    op = K.ResidualNorm(rows, width, [0, rows - LAST, rows], K.KNAP_NORM_LAYER, weight, K.KNAP_NORM_RMS, post_weight, ALPHA, EPS, dtype, dtype)
    op.forward(x, f, gate, scale, shift)
    op.backward(x, f, dx_out, dy, gate, scale, shift)
    torch.cuda.synchronize()
    one = {k: f64(v[1:]) for k, v in (("gate", gate), ("scale", scale), ("shift", shift))}
    val, bound = R.residual_norm(f64(x[-LAST:]), f64(f[-LAST:]), np.array([0, LAST]), R.LAYER, R.RMS, ALPHA, EPS, weight=f64(weight),
                                 post_weight=f64(post_weight), dx_out=f64(dx_out[-LAST:]), dy=f64(dy[-LAST:]), half_x=HALF[name], half_b=HALF[name],
                                 **one)
    for n, t in (("x_out", op.x_out), ("y", op.y), ("dx", op.dx), ("df", op.df)):
        assert np.all(np.abs(f64(t[-LAST:]) - val[n]) <= bound[n]), n
        assert not bool(t[:-LAST].any()), n
    for i, n in enumerate(("mean", "rstd", "post_mean", "post_rstd")):
        if n in val:
            assert np.all(np.abs(f64(op.stats[i, -LAST:]) - val[n]) <= bound[n]), n
    for n, t in (("dgate", op.dgate), ("dscale", op.dscale), ("dshift", op.dshift)):
        assert np.all(np.abs(f64(t[1:]) - val[n]) <= bound[n]), n
        assert not bool(t[0].any()), n
    for n, t in (("dweight", op.dweight), ("dpost_weight", op.dpost_weight)):
        assert np.all(np.abs(f64(t) - val[n]) <= bound[n]), n


@pytest.mark.gpu
def test_feed_forward_of_many_tokens():
    import torch
    import paper_2508_06001_amd as K
    T, D, F = 530_001, 64, 4104
    say(f"[gpu] large ffn T={T} D={D} F={F}")
    g = torch.Generator(device="cuda").manual_seed(7)
    new = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    wg, wu, wd = (new(F, D) / D ** 0.5).bfloat16(), (new(F, D) / D ** 0.5).bfloat16(), (new(D, F) / F ** 0.5).bfloat16()
    x, dy = (torch.zeros((T, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in (x, dy):
        t[-LAST:] = new(LAST, D).bfloat16()
    op = K.GatedFeedForward(T, D, F, wg, wu, wd)
    assert op.h.numel() * 2 > 2 ** 32
    op.forward(x)
    op.backward(x, dy)
    torch.cuda.synchronize()
    val, off = G.gated_ffn(*(t.double() for t in (x[-LAST:], wg, wu, wd)), False, dy[-LAST:].double())
    for n, t in (("gate", op.gate), ("up", op.up), ("h", op.h), ("y", op.y), ("dx", op.dx)):
        assert G.worst_block(t[-LAST:], val[n], off[n]) <= 1.0, n
        assert not bool(t[:-LAST].any()), n
    for n, t in (("dw_gate", op.dw_gate), ("dw_up", op.dw_up), ("dw_down", op.dw_down)):
        assert G.worst_block(t, val[n], off[n]) <= 1.0, n


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 24, 40])
def test_feed_forward_of_large_weights(T):
    """The last hidden units alone have weights, so that the oracle forms them alone; past 32 tokens with the gradients."""
    import torch
    import paper_2508_06001_amd as K
    D, F, units, train = 32776, 65536, 24, T > 32
    say(f"[gpu] large ffn T={T} D={D} F={F}")
    g = torch.Generator(device="cuda").manual_seed(8 + T)
    new = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    wg, wu = (torch.zeros((F, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    wd = torch.zeros((D, F), dtype=torch.bfloat16, device="cuda")
    assert wd.numel() * 2 > 2 ** 32
    for w in (wg, wu):
        w[-units:] = (new(units, D) / D ** 0.5).bfloat16()
    wd[:, -units:] = (new(D, units) / units ** 0.5).bfloat16()
    x, dy = new(T, D).bfloat16(), new(T, D).bfloat16()
    op = K.GatedFeedForward(T, D, F, wg, wu, wd, train=train)
    op.forward(x)
    if train:
        op.backward(x, dy)
    torch.cuda.synchronize()
    val, off = G.gated_ffn(*(t.double() for t in (x, wg[-units:], wu[-units:], wd[:, -units:].contiguous())), False, dy.double() if train else None)
    whole = {"y": op.y}
    tails = {"h": op.h}
    if train:
        whole["dx"] = op.dx
        tails.update(gate=op.gate, up=op.up, dw_down=op.dw_down)
        for n, t in (("dw_gate", op.dw_gate), ("dw_up", op.dw_up)):
            assert G.worst_block(t[-units:], val[n], off[n]) <= 1.0, n
            assert not bool(t[:-units].any()), n
    for n, t in whole.items():
        assert G.worst_block(t, val[n], off[n]) <= 1.0, n
    for n, t in tails.items():
        assert G.worst_block(t[:, -units:], val[n], off[n]) <= 1.0, n
        assert not bool(t[:, :-units].any()), n
