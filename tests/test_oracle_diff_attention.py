"""Pins of oracle/diff_attention.py: scalar loops, plain attention as its special cases, central differences, its own independence."""
import math

import numpy as np
import pytest

from oracle import attention as A
from oracle import diff_attention as D


def _bag(lens, H, d, seed):
    rng = np.random.default_rng(seed)
    cu = np.concatenate([[0], np.cumsum(lens)])
    q, k, v, do = rng.standard_normal((4, int(cu[-1]), H, d))
    return q, k, v, do, cu, rng.uniform(-0.5, 1.5, size=H)


@pytest.mark.parametrize("causal", [False, True])
def test_scalar_loops(causal):
    q, k, v, _, cu, lam = _bag([3, 0, 5, 1], 2, 4, 1)
    got, _ = D.diff_attn(q, k, v, cu, lam, 0.7, causal=causal)
    for s in range(4):
        for h in range(2):
            for i in range(cu[s], cu[s + 1]):
                seen = range(cu[s], i + 1 if causal else cu[s + 1])
                want = [0.0] * 4
                for m, f in ((0, 1.0), (1, -lam[h])):
                    e = [math.exp(0.7 * sum(q[i, h, 2 * m + c] * k[j, h, 2 * m + c] for c in range(2))) for j in seen]
                    assert got["lse"][m, h, i] == pytest.approx(math.log(sum(e)), rel=1e-12, abs=1e-12)
                    for c in range(4):
                        want[c] += f * sum(x * v[j, h, c] for x, j in zip(e, seen)) / sum(e)
                assert got["out"][i, h] == pytest.approx(want, rel=1e-11, abs=1e-12)


@pytest.mark.parametrize("causal", [False, True])
def test_no_second_map_is_plain_attention_of_half_the_columns(causal):
    """lam = 0: out and gradients are those of plain attention on q_1, k_1 with values of all d columns, which its oracle gives for d
    columns of q and k padded with zeros."""
    q, k, v, do, cu, _ = _bag([7, 4], 2, 8, 2)
    got, _ = D.diff_attn(q, k, v, cu, np.zeros(2), 0.5, do, causal)
    q0, k0 = q.copy(), k.copy()
    q0[..., 4:] = k0[..., 4:] = 0.0
    out, lse = A.varlen_attn_fwd(q0, k0, v, cu, 0.5, causal)
    dq, dk, dv = A.varlen_attn_bwd(q0, k0, v, cu, 0.5, do, causal)
    assert np.allclose(got["out"], out, atol=1e-13) and np.allclose(got["lse"][0], lse, atol=1e-13)
    assert np.allclose(got["dq"][..., :4], dq[..., :4], atol=1e-13) and np.allclose(got["dk"][..., :4], dk[..., :4], atol=1e-13)
    assert np.allclose(got["dv"], dv, atol=1e-13) and not got["dq"][..., 4:].any() and not got["dk"][..., 4:].any()


@pytest.mark.parametrize("causal", [False, True])
def test_central_differences(causal):
    q, k, v, do, cu, lam = _bag([4, 3], 1, 4, 3)
    got, _ = D.diff_attn(q, k, v, cu, lam, 0.6, do, causal)
    loss = lambda: (D.diff_attn(q, k, v, cu, lam, 0.6, None, causal)[0]["out"] * do).sum()  # noqa: E731
    for x, g in ((q, got["dq"]), (k, got["dk"]), (v, got["dv"]), (lam, got["dlam"])):
        for i in np.ndindex(x.shape):
            keep = x[i]
            x[i] = keep + 1e-5
            up = loss()
            x[i] = keep - 1e-5
            assert g[i] == pytest.approx((up - loss()) / 2e-5, rel=1e-6, abs=1e-8)
            x[i] = keep


def test_equal_maps_cancel_and_bounds_cover_a_rounded_run():
    q, k, v, do, cu, _ = _bag([6, 9], 2, 8, 4)
    q[..., 4:], k[..., 4:] = q[..., :4], k[..., :4]
    got, _ = D.diff_attn(q, k, v, cu, np.ones(2), 0.5, do)
    assert np.abs(got["out"]).max() < 1e-14 and np.abs(got["dv"]).max() < 1e-14
    assert np.allclose(got["dq"][..., :4], -got["dq"][..., 4:]) and np.allclose(got["dk"][..., :4], -got["dk"][..., 4:])
    # values moved by a relative 2^-9 (within the half step the bounds are for) stay inside
    rng = np.random.default_rng(5)
    lam = np.array([0.3, 0.8])
    got, bound = D.diff_attn(q, k, v, cu, lam, 0.5, do)
    for n in ("out", "out2", "dq", "dk", "dv"):
        assert np.all(np.abs(got[n] * 2.0 ** -9 * rng.uniform(-1, 1, got[n].shape)) <= bound[n])
