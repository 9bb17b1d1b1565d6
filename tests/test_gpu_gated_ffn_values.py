"""Gated feed-forward block on values at the ends of the range, on rows that are not finite, and between columns that are not: what a form's masks
behind the last row, column and k have to keep apart, at sizes that no stage divides, in every form of tiles."""
import pytest

from gpu_util import say
from oracle import gated_ffn as G
from test_gpu_gated_ffn import Guarded, inputs

HALF = 2.0 ** -8
# gate, up and dy of a column; x is a power of two, so that a and b are exact
FLAT = [(3e38, 1e-3, 0.03), (-3e38, 1e-3, 0.03), (1e37, 1e-3, 0.03), (-1e37, 1e-3, 0.03), (6.5e36, 1e-3, 0.03), (-6.5e36, 1e-3, 0.03), (1e30, 1e-3, 0.03),
        (-3e38, 1e-3, 4.0), (-1e38, 1e-3, 30.0),                   # dh a past the range, act(a) zero
        (-1e4, 1e20, 1e20), (-1e30, 3e38, 3e38),                   # dh b past the range, the slope zero
        (20.0, 1.0, 1.0), (-20.0, 1.0, 1.0), (17.0, 1.0, 1.0), (16.0, 1.0, 1.0), (-16.0, 1.0, 1.0), (0.5, 1.0, 1.0), (-0.5, 1.0, 1.0), (0.0, 1.0, 1.0)]


def of_single_columns(T, gelu, columns):
    import torch
    import paper_2508_06001_amd as K
    D = F = 64
    act = K.KNAP_GELU_TANH if gelu else K.KNAP_SILU
    col = torch.tensor((columns * D)[:D], device="cuda").bfloat16()
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


@pytest.mark.gpu
@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("T", [3, 24, 40, 300])
def test_where_the_activation_is_flat_its_gradients_are_what_the_formula_says(T, gelu):
    """Diagonal weights: every element by itself.  h, da, db and the result are rounded to bf16 once each, a half step for each; the logistic function has
    |a| 2^-23 of its value where it is small, below 2^-17 here; what is below 1e-36 may be zero."""
    say(f"[gpu] ffn, flat T={T} gelu={gelu}")
    of_single_columns(T, gelu, FLAT)


@pytest.mark.gpu
@pytest.mark.parametrize("gelu", [False, True])
def test_a_slope_above_one_at_the_end_of_the_range(gelu):
    """dh b slope is far inside the range, b slope is not; the same bounds."""
    say(f"[gpu] ffn, steep gelu={gelu}")
    of_single_columns(40, gelu, [(1.0, 3.3e38, 1e-10), (0.875, 3.38e38, -1e-10), (1.0, -3.38e38, 1e-20), (1.0, 1.0, 1.0)])


# one and two blocks of the few-token form, a row of tiles of 32 and of 64 tokens, the three forms of tiles, with parts and without, in every product
FORMS = [(5, 72, 136), (20, 72, 136), (33, 136, 72), (24, 4104, 4104), (60, 72, 136), (60, 1032, 2056), (300, 264, 136), (613, 1000, 2664), (4173, 1032, 5512),
         (5000, 1544, 264), (9000, 520, 2056), (12001, 1544, 4104)]


@pytest.mark.gpu
@pytest.mark.parametrize("T,D,F", FORMS)
def test_a_bad_row_stays_in_its_row_in_every_form(T, D, F):
    """The other rows have the same bits as without it: neither k's behind a row's end nor rows behind a tile's meet what the next row holds."""
    import torch
    import paper_2508_06001_amd as K
    say(f"[gpu] ffn, bad rows T={T} D={D} F={F}")
    x, wg, wu, wd, dy = inputs(T, D, F)
    f = K.GatedFeedForward(T, D, F, wg, wu, wd)
    y = f.forward(x).clone()
    dx = f.backward(x, dy)[0].clone()
    bad_x, bad_dy = {T - 1, T // 2}, {1, T // 2 + 1}
    bx, bdy = x.clone(), dy.clone()
    bx[T - 1] = float("nan")
    bx[T // 2, 0] = float("inf")
    bdy[1] = float("nan")
    bdy[T // 2 + 1, 0] = float("-inf")
    by = f.forward(bx).clone()
    bdx = f.backward(bx, bdy)[0].clone()
    torch.cuda.synchronize()
    for got, clean, bad in ((by, y, bad_x), (bdx, dx, bad_x | bad_dy)):
        good = torch.tensor([t not in bad for t in range(T)], device="cuda")
        assert torch.equal(got[good], clean[good])
        assert not bool(torch.isfinite(got[~good]).all(1).any())


@pytest.mark.gpu
@pytest.mark.parametrize("T,D,F", FORMS + [(17, 264, 520), (48, 264, 520), (64, 1032, 4104), (3000, 1536, 2056)])
def test_columns_between_rows_are_not_looked_at(T, D, F):
    """x and dy as columns of a wider tensor that is NaN elsewhere, y and dx as columns of another."""
    import torch
    import paper_2508_06001_amd as K
    say(f"[gpu] ffn, between NaN T={T} D={D} F={F}")
    x, wg, wu, wd, dy = inputs(T, D, F)
    wide = [Guarded(T, D, 24) for _ in range(4)]
    xs, dys, y, dx = (w.view for w in wide)
    xs.copy_(x)
    dys.copy_(dy)
    f = K.GatedFeedForward(T, D, F, wg, wu, wd)
    f.y, f.dx = y, dx
    f.forward(xs)
    f.backward(xs, dys)
    torch.cuda.synchronize()
    for n, w in zip(("x", "dy", "y", "dx"), wide):
        w.check(n)
    val, off = G.gated_ffn(*(t.double() for t in (x, wg, wu, wd)), False, dy.double())
    for n, t in (("y", y), ("dx", dx), ("dw_gate", f.dw_gate), ("dw_up", f.dw_up), ("dw_down", f.dw_down)):
        assert G.worst_block(t, val[n], off[n]) <= 1.0, n
