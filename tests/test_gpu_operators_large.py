"""Differential attention, rotary positions and layer norm on tensors of more than 2^32 bytes: rows behind that offset against the plain
definitions.  Bars as in the operators' own tests."""
import numpy as np
import pytest

from gpu_util import say
from oracle import diff_attention as D

T, H, d = 705_001, 24, 128        # 4.33e9 bytes a tensor
LAST = 501


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
def test_differential_attention(causal):
    import torch
    import paper_2508_06001_amd as K
    lens = [500] * 1409
    lens.append(T - sum(lens))
    assert lens[-1] == LAST
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    say(f"[gpu] large diff T={T} H={H} d={d} causal={causal}")
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k, v, dout = (torch.zeros((T, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(4))
    for t in (q, k, v, dout):
        t[-LAST:] = torch.randn((LAST, H, d), generator=g, device="cuda").bfloat16()
    lam = torch.linspace(-0.4, 1.3, H, device="cuda")
    scale = float(np.float32(0.125))
    attn = K.VarlenDiffAttention(cu, H, d, scale, lam, causal=causal)
    attn.forward(q, k, v)
    attn.backward(q, k, v, dout)
    torch.cuda.synchronize()
    heads = [0, H - 1]
    x = [f64(t[-LAST:, heads]) for t in (q, k, v)]
    want, bound = D.diff_attn(*x, np.array([0, LAST]), f64(lam)[heads], scale, f64(dout[-LAST:, heads]), causal)
    got = {"out": attn.out, "out2": attn.out2, "dq": attn.dq, "dk": attn.dk, "dv": attn.dv}
    for n, t in got.items():
        assert np.all(np.abs(f64(t[-LAST:, heads]) - want[n]) <= bound[n]), n
        assert not bool(t[:-LAST].any()), n            # everything else is zeros
    assert np.all(np.abs(f64(attn.lse[:, heads, -LAST:]) - want["lse"]) <= bound["lse"])
    assert np.all(np.abs(f64(attn.dlam[heads]) - want["dlam"]) <= bound["dlam"])       # zero rows add zeros


@pytest.mark.gpu
@pytest.mark.parametrize("rot", [128, 20])
def test_rotary_positions(rot):
    import torch
    import paper_2508_06001_amd as K
    say(f"[gpu] large rope T={T} rot={rot}")
    x = torch.zeros((T, H, d), dtype=torch.bfloat16, device="cuda")
    x[-LAST:] = torch.randn((LAST, H, d), generator=torch.Generator(device="cuda").manual_seed(6), device="cuda").bfloat16()
    y = torch.full_like(x, float("nan"))
    freq, factor = K.knap_rope_frequencies(rot)
    K.RotaryPositions(rot, K.KNAP_ROPE_HALF, freq, factor, cu_seqlens=[0, T]).forward(x, None, y, None)
    torch.cuda.synchronize()
    assert not bool(y[:-LAST].any())
    a = f64(x[-LAST:])
    ang = np.arange(T - LAST, T, dtype=np.float64)[:, None] * np.array(freq)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    h = rot // 2
    want = a.copy()
    want[..., :h], want[..., h:rot] = a[..., :h] * c - a[..., h:rot] * s, a[..., :h] * s + a[..., h:rot] * c
    near = 1e-6 * (np.abs(a[..., :h]) + np.abs(a[..., h:rot]))
    got = f64(y[-LAST:])
    off = np.abs(got - want)[..., :rot]
    assert np.all(off <= 2.0 ** -8 * np.abs(want)[..., :rot] + np.concatenate([near, near], -1) * (1 + 2.0 ** -8))
    assert np.array_equal(got[..., rot:], a[..., rot:])


@pytest.mark.gpu
@pytest.mark.parametrize("width", [1536, 1537])
def test_layer_norm(width):
    import torch
    import paper_2508_06001_amd as K
    rows, n = 1_400_001, 1000
    say(f"[gpu] large norm rows={rows} width={width}")
    g = torch.Generator(device="cuda").manual_seed(7)
    x, dy = (torch.zeros((rows, width), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in (x, dy):
        t[-n:] = torch.randn((n, width), generator=g, device="cuda").bfloat16()
    w, b = (torch.randn((width,), generator=g, device="cuda") for _ in range(2))
    norm = K.LayerNorm(rows, width, w, b)
    norm.forward(x)
    dx, dw, db = norm.backward(x, dy)
    torch.cuda.synchronize()
    a, e, ww = f64(x[-n:]), f64(dy[-n:]), f64(w)
    mean = a.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((a - mean) ** 2).mean(1, keepdims=True) + 1e-5)
    xh = (a - mean) * rstd
    gr = e * ww
    y = xh * ww + f64(b)
    want = rstd * (gr - gr.mean(1, keepdims=True) - xh * (gr * xh).mean(1, keepdims=True))
    # before the rounding to bf16: 32-bit arithmetic, far below 2^-16 of the largest terms
    assert np.all(np.abs(f64(norm.y[-n:]) - y) <= 2.0 ** -8 * np.abs(y) + 2.0 ** -16 * (np.abs(xh * ww) + np.abs(f64(b))))
    assert np.all(np.abs(f64(dx[-n:]) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -16 * rstd * (np.abs(gr) + np.abs(gr).max(1, keepdims=True) * (1 + np.abs(xh))))
    assert bool((norm.y[:-n] == b.bfloat16()).all()) and not bool(dx[:-n].any())
    # sums of n terms (the other rows add zeros) in any order: n 2^-24 of the sum of their magnitudes, and xh off by 2^-20
    for got, terms in ((dw, e * xh), (db, e)):
        assert np.all(np.abs(f64(got) - terms.sum(0)) <= (n * 2.0 ** -24 + 2.0 ** -18) * np.abs(terms).sum(0) + 1e-6)


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,d,rot,odd,given", [((1 << 27) + 11, 8, 8, False, False), ((1 << 24) + 5, 520, 2, True, True)])
def test_rotary_positions_of_more_tokens_than_one_grid_takes(tokens, d, rot, odd, given):
    """Eight tokens a workgroup, and one (rows on 2 bytes): more workgroups of 256 threads than 2^32 threads make.  In place, every row;
    the bar is that of test_gpu_rope.py."""
    import torch
    import paper_2508_06001_amd as K
    say(f"[gpu] large rope tokens={tokens} d={d} rot={rot} odd={odd} given={given}")
    g = torch.Generator(device="cuda").manual_seed(tokens)
    pad = 1 if odd else 0
    flat = torch.full((tokens * d + pad,), 3.0, dtype=torch.bfloat16, device="cuda")
    x = flat[pad:].view(tokens, 1, d)
    head = torch.randn((tokens, rot), generator=g, dtype=torch.bfloat16, device="cuda")
    x[:, 0, :rot] = head
    pos = torch.randint(0, 1 << 30, (tokens,), generator=g, dtype=torch.int32, device="cuda") if given else None
    freq, factor = K.knap_rope_frequencies(rot)
    rope = K.RotaryPositions(rot, K.KNAP_ROPE_INTERLEAVED, freq, factor, positions=pos, cu_seqlens=None if given else [0, tokens])
    rope.forward(x, None, x, None)
    torch.cuda.synchronize()
    f = torch.tensor(freq, dtype=torch.float64, device="cuda")
    for i in range(0, tokens, 1 << 24):
        rows = slice(i, min(tokens, i + (1 << 24)))
        p = (pos[rows] if given else torch.arange(rows.start, rows.stop, device="cuda")).double()
        ang = p[:, None] * f
        a, b = head[rows, 0::2].double(), head[rows, 1::2].double()
        near = (a.abs() + b.abs()) * (1e-6 + ang * 2.0 ** -51)
        got = x[rows, 0, :rot].double()
        for y, ref in ((got[:, 0::2], a * ang.cos() - b * ang.sin()), (got[:, 1::2], a * ang.sin() + b * ang.cos())):
            assert bool(((y - ref).abs() <= near + 2.0 ** -8 * (ref.abs() + near)).all()), i
    assert bool((x[:, 0, rot:] == 3.0).all())
