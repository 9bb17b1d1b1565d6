"""Gated feed-forward block on values at the ends of the range."""
import pytest

from gpu_util import say
from oracle import gated_ffn as G

HALF = 2.0 ** -8
# gate, up and dy of a column; x is a power of two, so that a and b are exact
FLAT = [(3e38, 1e-3, 0.03), (-3e38, 1e-3, 0.03), (1e37, 1e-3, 0.03), (-1e37, 1e-3, 0.03), (6.5e36, 1e-3, 0.03), (-6.5e36, 1e-3, 0.03), (1e30, 1e-3, 0.03),
        (-3e38, 1e-3, 4.0), (-1e38, 1e-3, 30.0),                   # dh a past the range, act(a) zero
        (-1e4, 1e20, 1e20), (-1e30, 3e38, 3e38),                   # dh b past the range, the slope zero
        (20.0, 1.0, 1.0), (-20.0, 1.0, 1.0), (17.0, 1.0, 1.0), (16.0, 1.0, 1.0), (-16.0, 1.0, 1.0), (0.5, 1.0, 1.0), (-0.5, 1.0, 1.0), (0.0, 1.0, 1.0)]


@pytest.mark.gpu
@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("T", [3, 24, 40, 300])
def test_where_the_activation_is_flat_its_gradients_are_what_the_formula_says(T, gelu):
    """Diagonal weights: every element by itself.  h, da, db and the result are rounded to bf16 once each, a half step for each; the logistic function has
    |a| 2^-23 of its value where it is small, below 2^-17 here; what is below 1e-36 may be zero."""
    import torch
    import paper_2508_06001_amd as K
    say(f"[gpu] ffn, flat T={T} gelu={gelu}")
    D = F = 64
    act = K.KNAP_GELU_TANH if gelu else K.KNAP_SILU
    col = torch.tensor((FLAT * 4)[:D], device="cuda").bfloat16()
    x = (0.5 ** (torch.arange(T, device="cuda") % 3)).float()[:, None].expand(T, D).bfloat16().contiguous()
    wg, wu = torch.diag(col[:, 0]).contiguous(), torch.diag(col[:, 1]).contiguous()
    wd = (0.5 * torch.eye(D, device="cuda")).bfloat16()
    dy = col[:, 2][None].expand(T, D).contiguous()
    f = K.GatedFeedForward(T, D, F, wg, wu, wd, act)
    y = f.forward(x)
    dx, dwg, dwu, _ = f.backward(x, dy)
    torch.cuda.synchronize()
    g, u, d, xv = (t.double() for t in (col[:, 0], col[:, 1], dy, x))
    a, b, dh = xv * g, xv * u, 0.5 * d
    value, slope = G.activation(a, gelu)
    da, db = dh * b * slope, dh * value
    da, db = (torch.where(t.abs() < 1e-100, torch.zeros_like(t), t) for t in (da, db))

    def near(got, want, size, roundings):
        ok = (got.double() - want).abs() <= (1.01 * roundings * HALF + 2.0 ** -17) * size + 1e-36
        # the sum of db of the largest column over 300 rows is 100 (1 + 1/4 + 1/16) 0.015 3e38 = 5.9e38, which bf16 holds as infinity
        past = want.abs() > 1.02 * float(torch.finfo(torch.bfloat16).max)
        return bool(torch.where(past, got.double() == torch.copysign(torch.full_like(want, float("inf")), want), ok).all())

    want = 0.5 * value * b
    assert near(y, want, want.abs(), 1)
    assert near(dx, da * g + db * u, (da * g).abs() + (db * u).abs(), 2)
    assert near(dwg, da.T @ xv, da.abs().T @ xv, 2)
    assert near(dwu, db.T @ xv, db.abs().T @ xv, 2)
