"""CPU oracle of differential attention over a packed bag, forward and backward.

TEST INFRASTRUCTURE ONLY, in float64, one (sequence, head) at a time, written from the definition:

    S_m = scale Q_m K_m^T  (Q_m, K_m: columns m d/2 .. (m + 1) d/2, m = 0, 1),  P_m = softmax rows of S_m,  O_m = P_m V
    out = O_0 - lam O_1,  lse_m = log sum exp of the rows of S_m
    dP = dO V^T,  dS_0 = P_0 (dP - rowsum(P_0 dP)),  dS_1 = -lam P_1 (dP - rowsum(P_1 dP))
    dQ_m = scale dS_m K_m,  dK_m = scale dS_m^T Q_m,  dV = (P_0 - lam P_1)^T dO,  dlam = -sum_ic dO_ic O_1,ic

Beside the values it returns how far a result may be off whose probabilities, score gradients and outputs are each rounded once to
`eps` relative (half a step of their type) and whose row sums dout . O_m are taken from rounded outputs: the sums of the magnitudes that the
roundings scale.  Probabilities times 2^15 in 16 bits with a step of 2^-24 at the lower end (fp16) are off by half of that, 2^-40 of a
probability, however small they are: `FLOOR`, which counts where no query pays a key more than about 2^-31.  Pins: tests/test_oracle_diff_attention.py."""
from __future__ import annotations

import numpy as np

FLOOR = 2.0 ** -40


def _one(Q, K, V, dO, lam, scale, causal, eps):
    L, d = Q.shape
    h = d // 2
    P, O, LSE, top = [], [], [], []
    for m in (0, 1):
        S = scale * (Q[:, m * h:(m + 1) * h] @ K[:, m * h:(m + 1) * h].T)
        size = scale * (np.abs(Q[:, m * h:(m + 1) * h]) @ np.abs(K[:, m * h:(m + 1) * h]).T)
        if causal:
            hidden = np.arange(L)[None, :] > np.arange(L)[:, None]
            S[hidden] = -np.inf
            size[hidden] = 0.0
        big = S.max(axis=1, keepdims=True)
        E = np.exp(S - big)
        total = E.sum(axis=1, keepdims=True)
        P.append(E / total)
        LSE.append((big + np.log(total))[:, 0])
        O.append(P[m] @ V)
        top.append(size.max(axis=1))
    r = {"out": O[0] - lam * O[1], "out2": O[1], "lse": np.stack(LSE)}
    aV, w = np.abs(V), abs(lam)
    off2 = (P[1] @ aV) * eps
    off = (P[0] @ aV) * eps + w * off2
    b = {"out": off + eps * (np.abs(r["out"]) + off), "out2": off2 + eps * (np.abs(O[1]) + off2)}
    b["lse"] = np.stack([t * 2.0 ** -18 + (32 + L / 32) * 2.0 ** -24 + np.abs(x) * 2.0 ** -22 + 2.0 ** -20 for t, x in zip(top, LSE)])
    if dO is None:
        return r, b
    dP = dO @ V.T
    adP = np.abs(dO) @ aV.T
    D = [(P[m] * dP).sum(axis=1, keepdims=True) for m in (0, 1)]
    e2 = (np.abs(dO) * b["out2"]).sum(axis=1, keepdims=True)
    eD = [(np.abs(dO) * b["out"]).sum(axis=1, keepdims=True) + w * e2, e2]
    soft = [t[:, None] * 2.0 ** -17 + 2.0 ** -15 for t in top]          # relative, of a probability formed in 32 bits
    dQ, dK = np.empty_like(Q), np.empty_like(K)
    bQ, bK = np.empty_like(Q), np.empty_like(K)
    for m, f in ((0, 1.0), (1, -lam)):
        cols = slice(m * h, (m + 1) * h)
        dS = f * P[m] * (dP - D[m])
        eS = np.abs(dS) * (2 * eps + soft[m]) + abs(f) * (P[m] * (eD[m] + adP * 2.0 ** -18) + FLOOR * np.abs(dP - D[m]))
        dQ[:, cols], dK[:, cols] = scale * (dS @ K[:, cols]), scale * (dS.T @ Q[:, cols])
        bQ[:, cols], bK[:, cols] = scale * (eS @ np.abs(K[:, cols])), scale * (eS.T @ np.abs(Q[:, cols]))
    W = P[0] - lam * P[1]
    r.update(dq=dQ, dk=dK, dv=W.T @ dO, dlam=-(dO * O[1]).sum())
    eW = np.abs(W) * eps + (P[0] * (soft[0] + 2.0 ** -11) + w * P[1] * (soft[1] + 2.0 ** -11))
    seen = np.tri(L) if causal else np.ones((L, L))
    bV = (eW + (1 + w) * FLOOR * seen).T @ np.abs(dO)
    b.update(dq=bQ + eps * (np.abs(dQ) + bQ), dk=bK + eps * (np.abs(dK) + bK), dv=bV + eps * (np.abs(r["dv"]) + bV),
             dlam=((P[1] * adP) * (soft[1] + L * 2.0 ** -24)).sum())
    return r, b


def diff_attn(q, k, v, cu_seqlens, lam, scale, dout=None, causal=False, eps=2.0 ** -8):
    """q, k, v, dout (T, H, d), lam (H,).  Returns two dicts of float64 arrays, the values and their bounds: out, out2 (T, H, d), lse
    (2, H, T) and, with dout, dq, dk, dv, dlam (H,)."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    T, H, d = q.shape
    names = ["out", "out2"] + (["dq", "dk", "dv"] if dout is not None else [])
    value = {n: np.zeros((T, H, d)) for n in names}
    bound = {n: np.zeros((T, H, d)) for n in names}
    for r in (value, bound):
        r["lse"] = np.zeros((2, H, T))
        if dout is not None:
            r["dlam"] = np.zeros(H)
    for s in range(len(cu_seqlens) - 1):
        a, e = int(cu_seqlens[s]), int(cu_seqlens[s + 1])
        if e <= a:
            continue
        for h in range(H):
            one = _one(q[a:e, h], k[a:e, h], v[a:e, h], None if dout is None else np.asarray(dout[a:e, h], dtype=np.float64), float(lam[h]), scale,
                       causal, eps)
            for whole, part in zip((value, bound), one):
                for n in names:
                    whole[n][a:e, h] = part[n]
                whole["lse"][:, h, a:e] = part["lse"]
                if dout is not None:
                    whole["dlam"][h] += part["dlam"]
    return value, bound
