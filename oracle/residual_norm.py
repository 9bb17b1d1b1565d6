"""The norms around a branch with its gate, residual scale and the next branch's modulation, forward and backward, in 64 bits, with a bound
for each result of a run that computes in 32 bits and rounds once at the end.

Bounds.  A 32-bit sum over the columns of a row (a thread's 32 values one after the other, then a tree) is off by less than 2^-18 of its
magnitudes, and with it (A = rstd max|v| of a row, as for layer norm) a normed value by A 2^-17 + |vh| 2^-18.  What goes into a norm with an
error of E moves the normed values by rstd E (2 + |vh|) at most (the value itself, the mean, rstd).  The rest follows term by term; every
product and sum of 32 bits adds 2^-24 of its value, for which 2^-21 stands where several meet.  Sums over the rows of a sequence run in a
workgroup's share one after the other and in 512 shares at most: with up to 100 rows of a share and the tree 2^-16 of the magnitudes."""
from __future__ import annotations

from typing import Dict, List, Optional, Tuple

import numpy as np

NONE, RMS, LAYER = 0, 1, 2


def normed(v: np.ndarray, kind: int, eps: float) -> Tuple[np.ndarray, np.ndarray, np.ndarray]:
    """Mean (zeros in an RMS norm), rstd and the normed rows."""
    mean = v.mean(1) if kind == LAYER else np.zeros(v.shape[0])
    c = v - mean[:, None]
    rstd = 1.0 / np.sqrt((c * c).mean(1) + eps)
    return mean, rstd, c * rstd[:, None]


def normed_back(g: np.ndarray, vh: np.ndarray, rstd: np.ndarray, kind: int) -> np.ndarray:
    out = g - vh * (g * vh).mean(1, keepdims=True)
    if kind == LAYER:
        out = out - g.mean(1, keepdims=True)
    return rstd[:, None] * out


def row_sequences(cu: np.ndarray) -> np.ndarray:
    return np.repeat(np.arange(len(cu) - 1), np.diff(cu))


def per_sequence(values: np.ndarray, cu: np.ndarray) -> np.ndarray:
    return np.stack([values[cu[s]:cu[s + 1]].sum(0) for s in range(len(cu) - 1)]) if len(cu) > 1 else np.zeros((0, values.shape[1]))


def residual_norm(x, f, cu, norm: int, post_norm: int, alpha: float, eps: float, weight=None, post_weight=None, gate=None, scale=None, shift=None,
                  dx_out=None, dy=None, half_x: float = 0.0, half_b: float = 0.0) -> Tuple[Dict[str, np.ndarray], Dict[str, np.ndarray]]:
    """Values and bounds of x_out, y, stats (mean, rstd, post_mean, post_rstd) and, where dx_out or dy is given, the gradients.  half_x, half_b:
    half a step of the types of x and of the branch.  All rows belong to a sequence of cu."""
    rows, width = x.shape
    seq = row_sequences(cu)
    ones = np.ones(width)
    w = ones if weight is None else weight
    wp = ones if post_weight is None else post_weight
    G = np.ones((rows, width)) if gate is None else gate[seq]
    S = np.ones((rows, width)) if scale is None else 1.0 + scale[seq]
    H = np.zeros((rows, width)) if shift is None else shift[seq]
    val: Dict[str, np.ndarray] = {}
    bound: Dict[str, np.ndarray] = {}
    col = lambda v: v[:, None]  # noqa: E731
    top = lambda v: np.abs(v).max(1, keepdims=True)  # noqa: E731

    # the branch
    xo, ex = x, np.zeros((rows, width))
    fh = efh = rp = af = None
    if f is not None:
        fh, efh, rp, af = f, np.zeros((rows, width)), np.ones(rows), 0.0
        if post_norm != NONE:
            m, rp, fh = normed(f, post_norm, eps)
            af = col(rp) * top(f)
            efh = af * 2.0 ** -17 + np.abs(fh) * 2.0 ** -18
            val["post_mean"], bound["post_mean"] = m, 2.0 ** -18 * np.abs(f).mean(1) + 2.0 ** -24 * np.abs(m)
            val["post_rstd"], bound["post_rstd"] = rp, 2.0 ** -16 * rp * (1 + af[:, 0] * 2.0 ** -6)
        gz = alpha * G * wp
        z = gz * fh
        xo = x + z
        ex = np.abs(gz) * efh + 2.0 ** -21 * (np.abs(z) + np.abs(x))
        val["x_out"], bound["x_out"] = xo, ex + half_x * (np.abs(xo) + ex)
    if norm != NONE:
        m, r, xh = normed(xo, norm, eps)
        a = col(r) * top(xo)
        exh = a * 2.0 ** -17 + np.abs(xh) * 2.0 ** -18 + col(r) * top(ex) * (2 + np.abs(xh))
        val["mean"], bound["mean"] = m, 2.0 ** -18 * np.abs(xo).mean(1) + 2.0 ** -24 * np.abs(m) + ex.max(1)
        val["rstd"], bound["rstd"] = r, r * (2.0 ** -16 * (1 + a[:, 0] * 2.0 ** -6) + 2 * r * ex.max(1))
        y = xh * w * S + H
        ey = np.abs(w * S) * exh + 2.0 ** -21 * (np.abs(xh * w * S) + np.abs(H))
        val["y"], bound["y"] = y, ey + half_b * (np.abs(y) + ey)
    if dx_out is None and dy is None:
        return val, bound

    X, eX = (np.zeros((rows, width)) if dx_out is None else dx_out.copy()), np.zeros((rows, width))
    if norm != NONE:
        g = dy * S * w
        gm, xm = top(g), top(xh)
        X = X + normed_back(g, xh, r, norm)
        # two means of products of g and xh, and xh in front of the second
        eX = col(r) * gm * ((1 + a) ** 2 * 2.0 ** -16 + (1 + np.abs(xh)) * 2 * top(exh) * (1 + 0 * xm))
        val["dshift"], bound["dshift"] = per_sequence(dy, cu), per_sequence(np.abs(dy), cu) * 2.0 ** -16
        eb = np.abs(dy) * (exh + np.abs(xh) * 2.0 ** -16)
        val["dscale"], bound["dscale"] = w * per_sequence(dy * xh, cu), np.abs(w) * per_sequence(eb, cu)
        val["dweight"], bound["dweight"] = (S * dy * xh).sum(0), (np.abs(S) * eb).sum(0) + 2.0 ** -16 * np.abs(S * dy * xh).sum(0)
    eX = eX + 2.0 ** -21 * np.abs(X) + (0 if dx_out is None else 2.0 ** -21 * np.abs(dx_out))
    val["dx"], bound["dx"] = X, eX + half_x * (np.abs(X) + eX)
    if f is not None:
        ec = eX * np.abs(fh) + np.abs(X) * efh + np.abs(X * fh) * 2.0 ** -16
        val["dgate"], bound["dgate"] = alpha * wp * per_sequence(X * fh, cu), np.abs(alpha * wp) * per_sequence(ec, cu)
        val["dpost_weight"] = (alpha * G * X * fh).sum(0)
        bound["dpost_weight"] = (np.abs(alpha * G) * ec).sum(0) + 2.0 ** -16 * np.abs(alpha * G * X * fh).sum(0)
        e = gz * X
        ee = np.abs(gz) * eX + 2.0 ** -21 * np.abs(e)
        if post_norm == NONE:
            df, edf = e, ee
        else:
            df = normed_back(e, fh, rp, post_norm)
            em = top(e)
            edf = col(rp) * (ee + top(ee) * (1 + np.abs(fh)) + em * (2 * efh + np.abs(fh) * top(efh)) + em * (1 + af) ** 2 * 2.0 ** -16)
        val["df"], bound["df"] = df, edf + half_b * (np.abs(df) + edf)
    return val, bound


def loss(args: Dict[str, Optional[np.ndarray]], cu, norm: int, post_norm: int, alpha: float, eps: float, dx_out, dy) -> float:
    """sum(dx_out x_out) + sum(dy y), whose gradients the backward returns."""
    val, _ = residual_norm(args["x"], args.get("f"), cu, norm, post_norm, alpha, eps, **{k: args.get(k) for k in NAMES})
    total = 0.0
    if dx_out is not None:
        total += float((dx_out * val.get("x_out", args["x"])).sum())
    if dy is not None:
        total += float((dy * val["y"]).sum())
    return total


NAMES: List[str] = ["weight", "post_weight", "gate", "scale", "shift"]
GRADIENT_OF = {"x": "dx", "f": "df", "weight": "dweight", "post_weight": "dpost_weight", "gate": "dgate", "scale": "dscale", "shift": "dshift"}
