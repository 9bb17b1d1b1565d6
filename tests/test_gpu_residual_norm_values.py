"""Residual norm without a norm in front of the next branch (a block's last residual): its gradients do not depend on x, nor dx and dgate on gate."""
import pytest

from gpu_util import say
from oracle import residual_norm as R
from test_gpu_residual_norm import BAGS, TYPES, call, check, make


@pytest.mark.gpu
@pytest.mark.parametrize("post", [R.NONE, R.RMS, R.LAYER])
@pytest.mark.parametrize("xt,bt", TYPES)
@pytest.mark.parametrize("width", [64, 128, 264, 1001, 1536, 5000, 9600])
def test_without_a_norm_bad_values_of_x_and_gate_reach_no_gradient_that_has_neither(width, xt, bt, post):
    import torch
    say(f"[gpu] residual norm, last residual width={width} {xt} {bt} post={post}")
    bag = BAGS["some"]
    c = make(bag, width, xt, bt, norm=R.NONE, post=post)
    clean = {k: v.clone() for k, v in call(c).items()}
    check(c, clean)
    assert torch.equal(clean["dx"], c["dx_out"])
    nan, inf = float("nan"), float("inf")
    c["x"][5, 3], c["x"][12, 0] = inf, nan
    c["x"][9] = nan
    c["gate"][2, 1] = inf                     # of rows 3 to 9
    got = call(c)
    for k in ("dx", "dgate"):
        assert torch.equal(got[k], clean[k]), k
    rows = torch.ones((sum(bag),), dtype=torch.bool, device="cuda")
    rows[3:10] = False
    columns = torch.arange(width, device="cuda") != 1
    assert torch.equal(got["df"][rows], clean["df"][rows])
    assert torch.equal(got["dpost_weight"][columns], clean["dpost_weight"][columns])
