"""Gated feed-forward block, forward and backward, in 64 bits, and how far a run may be off that multiplies bf16 operands, adds up in 32 bits and
rounds a, b, h, da, db and its results to bf16.

What is compared is blocks of up to 32 x 32 results by their 2-norm.  Every rounding to bf16 moves a value by up to 2^-8 of it, up or down as its
bits fall; in a sum over many products such errors add up as their squares do, and to `roundings` independent ones belongs sqrt(roundings) 2^-8
of the 2-norm that the result would have if its terms had independent signs - which is what the terms' norm below is: the square root of the
sum of their squares.  (2^-8 is the largest of each, 0.42 of that the usual one: no block comes near by chance.)  32-bit sums of K products are off by less
than K 2^-23 of the sum of their magnitudes."""
from __future__ import annotations

import math
from typing import Dict, Tuple

import torch

HALF = 2.0 ** -8


def activation(a: torch.Tensor, gelu: bool) -> Tuple[torch.Tensor, torch.Tensor]:
    """act(a) and its derivative."""
    if gelu:
        k = 2.0 * math.sqrt(2.0 / math.pi)
        u, du = k * (a + 0.044715 * a ** 3), k * (1 + 3 * 0.044715 * a * a)
    else:
        u, du = a, torch.ones_like(a)
    s = torch.sigmoid(u)
    slope = torch.where((s > 0) & (s < 1), a * du * s * (1 - s), torch.zeros_like(a)) + s
    return a * s, slope


def gated_ffn(x, wg, wu, wd, gelu: bool, dy=None) -> Tuple[Dict[str, torch.Tensor], Dict[str, torch.Tensor]]:
    """Results, and for each the root of the sum of squares of the terms whose errors it collects, times their bound."""
    a, b = x @ wg.T, x @ wu.T
    act, slope = activation(a, gelu)
    h = act * b
    val = {"gate": a, "up": b, "h": h, "y": h @ wd.T}
    K = {"gate": x.shape[1], "up": x.shape[1], "h": x.shape[1], "y": wd.shape[1]}
    e32 = lambda k, p, q: k * 2.0 ** -23 * (p.abs() @ q.abs())  # noqa: E731
    ea, eb = e32(K["gate"], x, wg.T), e32(K["up"], x, wu.T)
    eh = 1.2 * ea * b.abs() + eb * act.abs() + 2.0 ** -20 * h.abs()
    off = {"gate": ea + HALF * a.abs(), "up": eb + HALF * b.abs(), "h": eh + HALF * h.abs()}
    root = lambda e, w: torch.sqrt((e * e) @ (w * w))  # noqa: E731
    off["y"] = root(off["h"], wd.T) + e32(K["y"], h, wd.T) + HALF * val["y"].abs()
    if dy is None:
        return val, off
    dh = dy @ wd
    da, db = dh * b * slope, dh * act
    edh = e32(wd.shape[0], dy, wd)
    # da and db of a and b as they are kept; the slope's own slope is below 0.9
    eda = torch.sqrt((dh * slope * off["up"]) ** 2 + (0.9 * dh * b * off["gate"]) ** 2 + (HALF * da) ** 2) + edh * (b * slope).abs() + 2.0 ** -19 * (dh * b).abs()
    edb = torch.sqrt((1.2 * dh * off["gate"]) ** 2 + (HALF * db) ** 2) + edh * act.abs() + 2.0 ** -20 * db.abs()
    val.update(dx=da @ wg + db @ wu, dw_gate=da.T @ x, dw_up=db.T @ x, dw_down=dy.T @ h)
    T, F = x.shape[0], wg.shape[0]
    off["dx"] = torch.sqrt((eda * eda) @ (wg * wg) + (edb * edb) @ (wu * wu)) + e32(2 * F, da, wg) + e32(2 * F, db, wu)
    off["dw_gate"] = root(eda.T, x) + e32(T, da.T, x)
    off["dw_up"] = root(edb.T, x) + e32(T, db.T, x)
    off["dw_down"] = torch.sqrt((dy * dy).T @ (off["h"] ** 2)) + e32(T, dy.T, h)
    for n in ("dx", "dw_gate", "dw_up", "dw_down"):
        off[n] = off[n] + HALF * val[n].abs()
    return val, off


def worst_block(got: torch.Tensor, want: torch.Tensor, off: torch.Tensor, size: int = 32) -> float:
    """The largest over blocks of size x size of the 2-norm of the difference over that of the bound."""
    rows, cols = want.shape
    pad = (0, -cols % size, 0, -rows % size)
    of = lambda t: torch.nn.functional.pad(t.double() ** 2, pad).view(-(-rows // size), size, -(-cols // size), size).sum((1, 3)).sqrt()  # noqa: E731
    diff, bound = of(got.double() - want), of(off)
    assert bool(torch.isfinite(diff).all())
    return float(torch.where(bound > 0, diff / bound, torch.where(diff > 0, math.inf, 0.0)).max()) if diff.numel() else 0.0
