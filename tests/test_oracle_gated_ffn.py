"""The oracle of the gated feed-forward block: its gradients against automatic differentiation and differences of the plain formula, its bounds
against a run that rounds as the kernels do, and against planted mistakes."""
import pytest
import torch

from oracle import gated_ffn as G


def inputs(seed, T, D, F, dtype=torch.float64):
    g = torch.Generator().manual_seed(seed)
    new = lambda *s: torch.randn(s, generator=g, dtype=torch.float32)  # noqa: E731
    t = [new(T, D), new(F, D) / D ** 0.5, new(F, D) / D ** 0.5, new(D, F) / F ** 0.5, new(T, D)]
    return [v.bfloat16().to(dtype) for v in t]


def plain(x, wg, wu, wd, gelu):
    a = x @ wg.T
    act = torch.nn.functional.gelu(a, approximate="tanh") if gelu else torch.nn.functional.silu(a)
    return (act * (x @ wu.T)) @ wd.T


@pytest.mark.parametrize("gelu", [False, True])
def test_gradients_are_those_of_the_plain_formula(gelu):
    x, wg, wu, wd, dy = inputs(1, 5, 6, 7)
    val, _ = G.gated_ffn(x, wg, wu, wd, gelu, dy)
    leaves = [t.clone().requires_grad_(True) for t in (x, wg, wu, wd)]
    y = plain(*leaves, gelu)
    assert torch.allclose(y, val["y"], rtol=1e-12, atol=1e-12)
    for got, want in zip((val["dx"], val["dw_gate"], val["dw_up"], val["dw_down"]), torch.autograd.grad(y, leaves, dy)):
        assert torch.allclose(got, want, rtol=1e-11, atol=1e-12)
    h = 1e-5
    for i in range(3):
        up, down = x.clone(), x.clone()
        up[i, i] += h
        down[i, i] -= h
        diff = float(((plain(up, wg, wu, wd, gelu) - plain(down, wg, wu, wd, gelu)) * dy).sum() / (2 * h))
        assert abs(diff - float(val["dx"][i, i])) <= 1e-7 * (1 + abs(diff))


def rounded(x, wg, wu, wd, gelu, dy):
    """As the kernels round: 32-bit products of bf16 operands, a, b, h, da, db and results in bf16."""
    r = lambda t: t.bfloat16().float()  # noqa: E731
    x, wg, wu, wd, dy = (t.float() for t in (x, wg, wu, wd, dy))
    a, b = x @ wg.T, x @ wu.T
    h = r(G.activation(a, gelu)[0] * b)
    a, b = r(a), r(b)
    act, slope = G.activation(a, gelu)
    dh = dy @ wd
    da, db = r(dh * b * slope), r(dh * act)
    out = {"gate": a, "up": b, "h": h, "y": h @ wd.T, "dx": da @ wg + db @ wu, "dw_gate": da.T @ x, "dw_up": db.T @ x, "dw_down": dy.T @ h}
    return {n: r(t) for n, t in out.items()}


@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("T,D,F", [(1, 8, 8), (33, 136, 200), (200, 264, 72)])
def test_bounds_hold_for_a_rounded_run_and_not_for_mistakes(T, D, F, gelu):
    x, wg, wu, wd, dy = inputs(2, T, D, F)
    val, off = G.gated_ffn(x, wg, wu, wd, gelu, dy)
    got = rounded(x, wg, wu, wd, gelu, dy)
    for n in val:
        assert G.worst_block(got[n], val[n], off[n]) <= 1.0, n
    if T == 1:
        return
    for n in val:       # a unit of 8 columns left as zeros, two rows swapped
        wrong = got[n].clone()
        wrong[-1, -8:] = 0
        assert G.worst_block(wrong, val[n], off[n]) > 1.0, n
        wrong = got[n].clone()
        wrong[:2] = got[n][:2].flip(0)
        assert G.worst_block(wrong, val[n], off[n]) > 1.0, n
    # eight of the k's left out of a sum
    wrong = x[:, :-8].float() @ wg[:, :-8].T.float()
    assert G.worst_block(wrong, val["gate"], off["gate"]) > 1.0
