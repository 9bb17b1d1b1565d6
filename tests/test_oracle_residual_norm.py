"""The oracle of the residual norm: its gradients against central differences of its own forward, and its bounds against a run in 32 bits."""
import numpy as np
import pytest

from oracle import residual_norm as R

CU = np.array([0, 2, 2, 5])


def inputs(rng, f=True, rows=5, width=6, n=3):
    args = {"x": rng.standard_normal((rows, width)), "weight": rng.standard_normal(width), "post_weight": rng.standard_normal(width),
            "gate": rng.standard_normal((n, width)), "scale": rng.standard_normal((n, width)), "shift": rng.standard_normal((n, width))}
    if f:
        args["f"] = rng.standard_normal((rows, width))
    return args


@pytest.mark.parametrize("norm", [R.NONE, R.RMS, R.LAYER])
@pytest.mark.parametrize("post_norm", [R.NONE, R.RMS, R.LAYER])
@pytest.mark.parametrize("f", [True, False])
def test_gradients_are_those_of_the_forward(norm, post_norm, f):
    if not f and (norm == R.NONE or post_norm != R.NONE):
        pytest.skip("no such operator")
    rng = np.random.default_rng(3)
    args = inputs(rng, f)
    dx_out, dy = rng.standard_normal((2, 5, 6))
    if norm == R.NONE:
        dy = None
    names = ["x", "shift", "scale", "weight"] if norm != R.NONE else ["x"]
    names += ["f", "gate", "post_weight"] if f else []
    val, _ = R.residual_norm(args["x"], args.get("f"), CU, norm, post_norm, 0.7, 1e-3, **{k: args[k] for k in R.NAMES}, dx_out=dx_out, dy=dy)
    h = 1e-5
    for name in names:
        a, grad = args[name], val[R.GRADIENT_OF[name]]
        for i in np.ndindex(a.shape):
            keep = a[i]
            a[i] = keep + h
            up = R.loss(args, CU, norm, post_norm, 0.7, 1e-3, dx_out, dy)
            a[i] = keep - h
            diff = (up - R.loss(args, CU, norm, post_norm, 0.7, 1e-3, dx_out, dy)) / (2 * h)
            a[i] = keep
            # h^2 times third derivatives, which small rows raise to 1e4 at most here, and 2^-52 of a loss below 100 over h
            assert abs(diff - grad[i]) <= 1e-5 * (1 + abs(diff)), (name, i, diff, grad[i])


def test_a_sequence_without_rows_has_no_gradients_and_a_planted_mistake_passes_the_bounds():
    rng = np.random.default_rng(4)
    args = inputs(rng)
    dx_out, dy = rng.standard_normal((2, 5, 6))
    val, bound = R.residual_norm(args["x"], args["f"], CU, R.LAYER, R.RMS, 0.7, 1e-3, **{k: args[k] for k in R.NAMES}, dx_out=dx_out, dy=dy,
                                 half_x=2.0 ** -8, half_b=2.0 ** -8)
    for n in ("dgate", "dscale", "dshift"):
        assert not val[n][1].any()
    # the vectors of another sequence, and a mean left out
    other = {k: args[k][[1, 0, 2]] if k in ("gate", "scale", "shift") else args[k] for k in R.NAMES}
    for wrong, _ in (R.residual_norm(args["x"], args["f"], CU, R.LAYER, R.RMS, 0.7, 1e-3, **other, dx_out=dx_out, dy=dy),
                     R.residual_norm(args["x"], args["f"], CU, R.RMS, R.RMS, 0.7, 1e-3, **{k: args[k] for k in R.NAMES}, dx_out=dx_out, dy=dy),
                     R.residual_norm(args["x"], args["f"], CU, R.LAYER, R.LAYER, 0.7, 1e-3, **{k: args[k] for k in R.NAMES}, dx_out=dx_out, dy=dy)):
        for n in ("y", "dx", "df"):
            assert not np.all(np.abs(wrong[n] - val[n]) <= bound[n]), n
