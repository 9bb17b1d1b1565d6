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


def _bf16(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).bfloat16().double().numpy()


def _fp16(x):
    """Times 2^15 in fp16."""
    return (x * 2.0 ** 15).astype(np.float16).astype(np.float64) * 2.0 ** -15


def _rounded(q, k, v, do, cu, lam, scale, causal, drop=""):
    """The operator's steps with every rounding that its bounds are for: probabilities, score gradients and outputs to bf16, the probabilities of
    dK and dV to fp16 times 2^15 on the way, D_m from the rounded outputs.  `drop` leaves a term out or takes a wrong one."""
    T, H, d = q.shape
    h2 = d // 2
    r = {n: np.zeros((T, H, d)) for n in ("out", "out2", "dq", "dk", "dv")}
    r.update(lse=np.zeros((2, H, T)), dlam=np.zeros(H))
    for s in range(len(cu) - 1):
        a, e = int(cu[s]), int(cu[s + 1])
        for h in range(H):
            V, dO, w = v[a:e, h], do[a:e, h], lam[h]
            P, O = [], []
            for m in (0, 1):
                cols = slice(m * h2, (m + 1) * h2)
                S = scale * (q[a:e, h, cols] @ k[a:e, h, cols].T)
                if causal:
                    S[np.arange(e - a)[None, :] > np.arange(e - a)[:, None] + (drop == "one key behind the mask")] = -np.inf
                top = S.max(1, keepdims=True)
                E = np.exp(S - top)
                total = E.sum(1, keepdims=True)
                r["lse"][m, h, a:e] = (top + np.log(total))[:, 0]
                P.append(E / total)
                O.append(_bf16(E) @ V / total)
            sign = -1.0 if drop == "sign of lambda" else 1.0
            r["out"][a:e, h] = out = _bf16(O[0] - sign * (0.0 if drop == "second map" else w) * O[1])
            r["out2"][a:e, h] = out2 = _bf16(O[1])
            D2 = (dO * out2).sum(1, keepdims=True)
            D1 = (dO * out).sum(1, keepdims=True) + (0.0 if drop == "lambda in D_1" else w) * D2
            dP = dO @ V.T
            D = [0.0 if drop == "D_1" else D1, 0.0 if drop == "D_2" else D1 if drop == "D_1 for D_2" else D2]
            r["dlam"][h] -= (P[1] * dP).sum() if drop != "first map's dlambda" else (P[0] * dP).sum()
            for m, f in ((0, 1.0), (1, -(1.0 if drop == "lambda in dq and dk" else sign * w))):
                cols = slice(m * h2, (m + 1) * h2)
                by = 1.0 if drop == "scale" else scale
                dS = _bf16(P[m] * (dP - D[m]))
                r["dq"][a:e, h, cols] = _bf16(by * f * (dS @ k[a:e, h, cols]))
                dS = _bf16(_fp16(P[m]) * (dP - D[m]))
                r["dk"][a:e, h, cols] = _bf16(by * f * (dS.T @ q[a:e, h, cols]))
            W = P[0] if drop == "lambda in dv" else _fp16(P[0]) - sign * w * P[1]
            r["dv"][a:e, h] = _bf16(_bf16(W).T @ dO)
    return r


def _outside(got, want, bound):
    """Outputs with an element outside its bound."""
    return {n for n in got if bool((np.abs(got[n] - want[n]) > bound[n]).any())}


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens,d", [([40, 1, 90], 64), ([150], 128)])
def test_bounds_cover_the_roundings_and_no_missing_term(lens, d, causal):
    q, k, v, do, cu, _ = _bag(lens, 2, d, 6 + d)
    q, k, v, do = (_bf16(x) for x in (q, k, v, do))
    lam, scale = np.array([0.6, -0.4]), (d // 2) ** -0.5
    want, bound = D.diff_attn(q, k, v, cu, lam, scale, do, causal)
    args = (q, k, v, do, cu, lam, scale, causal)
    assert _outside(_rounded(*args), want, bound) == set()
    # (without lambda in D_1 dk stays inside at 150 rows, where its bound, a sum over the queries, has outgrown that term; dq shows it)
    reached = {"second map": {"out"}, "sign of lambda": {"out", "dq", "dk", "dv"}, "lambda in D_1": {"dq"}, "D_1": {"dq", "dk"}, "D_2": {"dq", "dk"},
               "D_1 for D_2": {"dq", "dk"}, "lambda in dq and dk": {"dq", "dk"}, "scale": {"dq", "dk"}, "lambda in dv": {"dv"},
               "first map's dlambda": {"dlam"}}
    if causal:
        reached["one key behind the mask"] = {"out", "out2", "lse", "dq", "dk", "dv", "dlam"}
    for drop, outputs in reached.items():
        assert outputs <= _outside(_rounded(*args, drop=drop), want, bound), drop
