"""Rotary positions against the formula in 64 bits: layouts, parts of the head, axes, strides, bags, far positions.

Bars.  A result is off by the rounding to bf16, half a step, 2^-8 of its value, and by what 32-bit arithmetic did before it: products
and sum of a pair 3 roundings (2^-24 each), the sine and cosine 2 ulp (2^-22), the fraction of a turn, rounded to 32 bits, half a turn times
2^-24 times 2 pi (2^-22.3); below 10^-6 (|a| + |b|) factor together.  The angle itself, in 64 bits, is off by three roundings of
2^-53 each relative to its size here and by one in the reference: 4 angle 2^-53 < angle 2^-51."""
import math

import numpy as np
import pytest

from gpu_util import say


def rope_ref(x, pos, freq, factor, rot, half, sign=1.0):
    """x (T, H, d) float64, pos (T, rot / 2) -> turned x, and the bound of what comes before the rounding."""
    ang = pos.astype(np.float64) * freq[None, :]
    c, s = (factor * np.cos(ang))[:, None, :], (sign * factor * np.sin(ang))[:, None, :]
    ia = np.arange(rot // 2) if half else 2 * np.arange(rot // 2)
    ib = ia + rot // 2 if half else ia + 1
    y, bound = x.copy(), np.zeros_like(x)
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
    near = (np.abs(a) + np.abs(b)) * abs(factor) * (1e-6 + np.abs(ang) * 2.0 ** -51)[:, None, :]
    bound[..., ia] = bound[..., ib] = near
    return y, bound


def close(got, ref, bound, what):
    err = np.abs(got - ref)
    assert np.all(err <= bound + 2.0 ** -8 * (np.abs(ref) + bound)), (what, float(np.max(err - bound - 2.0 ** -8 * (np.abs(ref) + bound))))


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


@pytest.mark.gpu
@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("T,H,Hk,d,rot", [(1, 1, 1, 64, 64), (1, 24, 24, 128, 128), (5, 2, 1, 128, 32), (67, 3, 2, 64, 20), (130, 2, 0, 128, 128),
                                          (333, 6, 6, 80, 80), (33, 4, 4, 10, 6), (1000, 12, 4, 64, 48), (257, 1, 1, 1024, 1024), (7, 5, 1, 2, 2),
                                          (4099, 3, 3, 128, 96), (9001, 1, 0, 1024, 1024)])
def test_turned_columns(T, H, Hk, d, rot, half, bwd):
    import torch
    import paper_2508_06001_amd as K
    say(f"[gpu] rope T={T} H={H}/{Hk} d={d} rot={rot} half={half} bwd={bwd}")
    g = torch.Generator(device="cuda").manual_seed(T + rot)
    q, k = (torch.randn((T, h, d), generator=g, device="cuda").bfloat16() for h in (H, max(Hk, 1)))
    k = k if Hk else None
    pos = torch.randint(0, 5000, (T,), generator=g, device="cuda", dtype=torch.int32)
    freq, factor = K.knap_rope_frequencies(rot, 10000.0, K.KNAP_ROPE_PARTS, 4.0, 512)
    guard = [torch.full((T + 2, h, d), float("nan"), dtype=torch.bfloat16, device="cuda") for h in (H, max(Hk, 1))]
    qo, ko = guard[0][1:-1], guard[1][1:-1] if Hk else None
    rope = K.RotaryPositions(rot, K.KNAP_ROPE_HALF if half else K.KNAP_ROPE_INTERLEAVED, freq, factor, positions=pos)
    (rope.backward if bwd else rope.forward)(q, k, qo, ko)
    torch.cuda.synchronize()
    p = np.repeat(pos.cpu().numpy()[:, None], rot // 2, 1)
    for x, y in ((q, qo),) + (((k, ko),) if Hk else ()):
        ref, bound = rope_ref(f64(x), p, np.array(freq), np.float32(factor).astype(np.float64), rot, half, -1.0 if bwd else 1.0)
        close(f64(y), ref, bound, "turned")
        assert torch.equal(y[..., rot:], x[..., rot:])
    for t in guard[: 2 if Hk else 1]:
        assert bool(torch.isnan(t[0]).all()) and bool(torch.isnan(t[-1]).all())
    for x, y in ((q, qo), (k, ko)):        # in place: the same bits
        if x is not None:
            z = x.clone()
            (rope.backward if bwd else rope.forward)(z, None, z, None)
            assert torch.equal(z, y)


@pytest.mark.gpu
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("lens,past", [([1], 0), ([0, 5, 0, 1, 300, 0], 0), ([37, 128, 200, 311], 9), ([0], 4), ([3] * 700 + [0] * 40, 3),
                                       ([1] * 2048, 0), ([5000], 17)])
def test_positions_of_a_bag(lens, past, half):
    """Positions in the own sequence; rows behind the last sequence stay as they were."""
    import torch
    import paper_2508_06001_amd as K
    T, H, d = sum(lens), 3, 64
    say(f"[gpu] rope bag n_seq={len(lens)} T={T} past={past} half={half}")
    g = torch.Generator(device="cuda").manual_seed(T)
    q, k = (torch.randn((T + past, H, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    qo, ko = (torch.full_like(q, 7.0) for _ in range(2))
    freq, factor = K.knap_rope_frequencies(d)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    K.RotaryPositions(d, K.KNAP_ROPE_HALF if half else K.KNAP_ROPE_INTERLEAVED, freq, factor, cu_seqlens=cu).forward(q, k, qo, ko)
    torch.cuda.synchronize()
    p = np.concatenate([np.arange(n) for n in lens]) if T else np.zeros(0, dtype=np.int64)
    for x, y in ((q, qo), (k, ko)):
        ref, bound = rope_ref(f64(x[:T]), np.repeat(p[:, None], d // 2, 1), np.array(freq), 1.0, d, half)
        close(f64(y[:T]), ref, bound, "bag")
        assert bool((y[T:] == 7.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("pairs", [[64], [8, 28, 28], [0, 64, 0, 0], [1, 61, 1, 1]])
def test_axes_and_far_positions(pairs, half):
    import torch
    import paper_2508_06001_amd as K
    T, H, d = 97, 2, 128
    say(f"[gpu] rope axes {pairs} half={half}")
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k = (torch.randn((T, H, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    pos = torch.randint(-(1 << 31), (1 << 31) - 1, (T, len(pairs)), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    pos[: T // 2] = pos[: T // 2] % 1000000
    freq = [f for n in pairs if n for f in K.knap_rope_frequencies(2 * n)[0]]
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    K.RotaryPositions(d, K.KNAP_ROPE_HALF if half else K.KNAP_ROPE_INTERLEAVED, freq, 1.0, positions=pos, axis_pairs=pairs).forward(q, k, qo, ko)
    torch.cuda.synchronize()
    p = np.repeat(pos.cpu().numpy(), pairs, axis=1)
    for x, y in ((q, qo), (k, ko)):
        ref, bound = rope_ref(f64(x), p, np.array(freq), 1.0, d, half)
        close(f64(y), ref, bound, "axes")


@pytest.mark.gpu
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("form", ["fused", "fused_last", "heads_first", "odd", "broadcast", "padded_out", "half_unit"])
def test_strides(form, half):
    """Slices of one projection, heads outside of tokens, rows that start on 2 bytes only, one head for all: the bits of contiguous tensors."""
    import torch
    import paper_2508_06001_amd as K
    T, H, d, rot = 45, 4, 64, 32
    say(f"[gpu] rope strides {form} half={half}")
    g = torch.Generator(device="cuda").manual_seed(9)
    new = lambda *shape: torch.randn(shape, generator=g, device="cuda").bfloat16()  # noqa: E731
    if form == "fused":
        qkv = new(T, 3, H, d)
        q, k = qkv[:, 0], qkv[:, 1]
    elif form == "fused_last":
        qkv = new(T, H, 3, d)
        q, k = qkv[:, :, 0], qkv[:, :, 1]
    elif form == "heads_first":
        q, k = new(H, T, d).transpose(0, 1), new(H, T, d).transpose(0, 1)
    elif form == "odd":
        q, k = new(T, H, d + 3)[..., 1:d + 1], new(T, H, d + 1)[..., :d]
    elif form == "half_unit":
        q, k = new(T, H, d + 4)[..., 4:], new(T, H, d)
    elif form == "broadcast":
        q, k = new(T, H, d), new(T, 1, d).expand(T, H, d)
    else:
        q, k = new(T, H, d), new(T, H, d)
    pos = torch.arange(T, device="cuda", dtype=torch.int32) * 11
    freq, _ = K.knap_rope_frequencies(rot, 500000.0)
    rope = K.RotaryPositions(rot, K.KNAP_ROPE_HALF if half else K.KNAP_ROPE_INTERLEAVED, freq, 1.25, positions=pos)
    want = [torch.empty((T, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    rope.forward(q.contiguous(), k.contiguous(), *want)
    if form == "padded_out":
        base = torch.full((H + 1, T, 2 * d), 3.0, dtype=torch.bfloat16, device="cuda")
        got = [base[:H, :, :d].transpose(0, 1), torch.empty_like(want[1])]
    else:
        got = [torch.empty_like(x) for x in want]
    rope.forward(q, k, *got)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    if form == "padded_out":
        assert bool((base[:H, :, d:] == 3.0).all()) and bool((base[H] == 3.0).all())
    if form != "broadcast":           # in place, in its own strides
        rope.forward(q, k, q, k)
        assert torch.equal(q, want[0]) and torch.equal(k, want[1])


@pytest.mark.gpu
def test_infinities_and_nan_stay_in_their_pair():
    import torch
    import paper_2508_06001_amd as K
    x = torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    x[1, 0, 5], x[1, 1, 40], x[2, 0, 60] = float("nan"), float("inf"), float("-inf")
    y = torch.empty_like(x)
    K.RotaryPositions(64, K.KNAP_ROPE_HALF, K.knap_rope_frequencies(64)[0], 1.0, cu_seqlens=[0, 3]).forward(x, None, y, None)
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    for t, h, c in ((1, 0, 5), (1, 1, 8), (2, 0, 28)):
        want[t, h, c] = want[t, h, c + 32] = True
    assert torch.equal(bad, want)


@pytest.mark.gpu
def test_backward_is_the_transpose_and_captured_calls_follow_their_inputs():
    import torch
    import paper_2508_06001_amd as K
    T, H, d = 200, 4, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, gq, gk = (torch.randn((T, H, d), generator=g, device="cuda").bfloat16() for _ in range(4))
    rope = K.RotaryPositions(d, K.KNAP_ROPE_INTERLEAVED, K.knap_rope_frequencies(d)[0], 1.0, cu_seqlens=[0, 77, 77, 200])
    out = [torch.empty_like(q) for _ in range(4)]
    rope.forward(q, k, out[0], out[1])
    rope.backward(gq, gk, out[2], out[3])
    torch.cuda.synchronize()
    for x, y, gy, gx in ((q, out[0], gq, out[2]), (k, out[1], gk, out[3])):
        # <R x, g> = <x, R^T g>, each side's rounded factor off by 2^-8 of itself at most, all of them independent signs
        a, b = (f64(y) * f64(gy)).sum(), (f64(x) * f64(gx)).sum()
        assert abs(a - b) <= 2.0 ** -8 * (np.abs(f64(y) * f64(gy)).sum() + np.abs(f64(x) * f64(gx)).sum())
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    buf = [torch.empty_like(q) for _ in range(2)]
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        rope.forward(q, k, *buf)
        rope.backward(buf[0], buf[1], buf[0], buf[1])
    for turn in range(3):
        q.normal_(generator=g)
        k.normal_(generator=g)
        graph.replay()
        eager = [torch.empty_like(q) for _ in range(2)]
        rope.forward(q, k, *eager)
        rope.backward(*eager, *eager)
        torch.cuda.synchronize()
        assert torch.equal(buf[0], eager[0]) and torch.equal(buf[1], eager[1]), turn


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
def test_attention_with_rotary_positions(causal):
    """VarlenAttention with rotary positions is the three calls one after the other, bit for bit, and its gradients are those of the
    turned attention (64-bit oracle)."""
    import torch
    import paper_2508_06001_amd as K
    from oracle import attention as A
    lens, H, d = [130, 1, 0, 75], 2, 64
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    T, scale = int(cu[-1]), 0.125
    g = torch.Generator(device="cuda").manual_seed(11)
    q, k, v, do = (torch.randn((T, H, d), generator=g, device="cuda").bfloat16() for _ in range(4))
    freq, _ = K.knap_rope_frequencies(d)
    rope = K.RotaryPositions(d, K.KNAP_ROPE_HALF, freq, 1.0, cu_seqlens=cu)
    attn = K.VarlenAttention(cu, H, d, scale, causal=causal, rope=rope)
    plain = K.VarlenAttention(cu, H, d, scale, causal=causal)
    out, _ = attn.forward(q, k, v)
    dq, dk, dv = attn.backward(q, k, v, do)
    qt, kt = torch.empty_like(q), torch.empty_like(k)
    rope.forward(q, k, qt, kt)
    want, _ = plain.forward(qt, kt, v)
    gq, gk, gv = plain.backward(qt, kt, v, do)
    rope.backward(gq, gk, gq, gk)
    torch.cuda.synchronize()
    for a, b in ((out, want), (dq, gq), (dk, gk), (dv, gv)):
        assert torch.equal(a, b)
    p = np.repeat(np.concatenate([np.arange(n) for n in lens])[:, None], d // 2, 1)
    turn = lambda x, sign: rope_ref(x, p, np.array(freq), 1.0, d, True, sign)[0]  # noqa: E731
    ref = A.varlen_attn_bwd(turn(f64(q), 1.0), turn(f64(k), 1.0), f64(v), cu, scale, f64(do), causal)
    for name, x, y in (("dq", dq, turn(ref[0], -1.0)), ("dk", dk, turn(ref[1], -1.0)), ("dv", dv, ref[2])):
        rel = np.linalg.norm(f64(x) - y) / np.linalg.norm(y)
        say(f"[parity] turned attention causal={causal} {name} rel={rel:.2e}")
        assert rel <= 3e-2 + 2 * 2.0 ** -8, name        # attention's bar, and the rounding of the turned q, k and of the gradient turned back


def test_frequencies_against_their_definitions():
    import paper_2508_06001_amd as K
    for rot in (2, 4, 20, 64, 128):
        plain, one = K.knap_rope_frequencies(rot, 10000.0)
        want = [10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]
        assert one == 1.0 and plain == pytest.approx(want, rel=1e-14)
        linear, one = K.knap_rope_frequencies(rot, 10000.0, K.KNAP_ROPE_LINEAR, 8.0)
        assert one == 1.0 and linear == pytest.approx([f / 8.0 for f in want], rel=1e-14)
        if rot > 2:
            base, one = K.knap_rope_frequencies(rot, 10000.0, K.KNAP_ROPE_BASE, 8.0)
            assert one == 1.0 and base[0] == 1.0 and base[-1] == pytest.approx(want[-1] / 8.0, rel=1e-12)
        parts, factor = K.knap_rope_frequencies(rot, 10000.0, K.KNAP_ROPE_PARTS, 8.0, 4096, 1.0, 32.0)
        assert factor == pytest.approx(0.1 * math.log(8.0) + 1.0, rel=1e-14)
        for f, got in zip(want, parts):
            turns = 4096 * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - 1.0) / 31.0))
            assert got == pytest.approx(keep * f + (1 - keep) * f / 8.0, rel=1e-13)


def test_bad_arguments_are_refused_without_touching_a_gpu():
    import ctypes as C
    import paper_2508_06001_amd as K
    f, bad = K.lib.knap_rope_fwd, K.KNAP_ERR_INVALID_ARG
    strides = lambda *s: (C.c_int64 * 8)(*s)  # noqa: E731
    ints = lambda *s: (C.c_int * len(s))(*s)  # noqa: E731

    def call(q=64, k=1 << 20, tokens=8, H=2, H_k=2, d=64, s=None, rot=64, layout=0, pos=64, axes=1, pairs=None, cu=0, n_seq=0, freq=64,
             factor=1.0, qo=2 << 20, ko=3 << 20):
        return f(q, k, tokens, H, H_k, d, s, rot, layout, pos, axes, pairs, cu, n_seq, freq, factor, qo, ko, 0)

    assert call(tokens=0) == K.KNAP_OK and call(pos=0, n_seq=0) == K.KNAP_OK
    assert call(tokens=0, q=0, k=0, freq=0, qo=0, ko=0) == K.KNAP_OK
    for wrong in (dict(tokens=-1), dict(tokens=1 << 31), dict(H=0), dict(H_k=-1), dict(d=0), dict(d=1026, rot=64), dict(rot=0), dict(rot=63),
                  dict(rot=66), dict(layout=2), dict(axes=0), dict(axes=5), dict(axes=2), dict(axes=2, pairs=ints(16, 15)),
                  dict(axes=2, pairs=ints(40, -8)), dict(axes=2, pairs=ints(32, 1)), dict(factor=float("nan")), dict(factor=float("inf")),
                  dict(q=0), dict(k=0), dict(qo=0), dict(ko=0), dict(freq=0), dict(q=65), dict(freq=68), dict(pos=66), dict(H=1 << 18, d=64),
                  dict(qo=3 << 20), dict(pos=0, n_seq=-1, cu=64), dict(pos=0, n_seq=1, cu=0),
                  dict(s=strides(128, 64, 128, 64, 127, 64, 128, 64)),          # rows of q_out overlap
                  dict(s=strides(128, 64, 128, 64, 128, 63, 128, 64)), dict(s=strides(128, 64, 128, 64, 128, 64, 0, 64)),
                  dict(s=strides(-128, 64, 128, 64, 128, 64, 128, 64)), dict(s=strides(128, 64, 128, 64, 64, 511, 128, 64)),
                  dict(qo=64, s=strides(128, 64, 128, 64, 256, 64, 128, 64))):   # in place with other strides
        assert call(**wrong) == bad, wrong
    assert call(pos=0, n_seq=K.KNAP_MAX_SEQS + 1, cu=64) == K.KNAP_ERR_TOO_MANY_SEQS
    for args in ((0, 1e4, 0, 1.0), (3, 1e4, 0, 1.0), (64, 0.0, 0, 1.0), (64, 1e4, 4, 1.0), (64, 1e4, -1, 1.0), (64, 1e4, 1, 0.5),
                 (64, float("nan"), 0, 1.0), (2, 1e4, K.KNAP_ROPE_BASE, 2.0), (64, 1e4, 1, float("inf")), (4, 1e4, K.KNAP_ROPE_BASE, 1e160)):
        with pytest.raises(K.KnapError):
            K.knap_rope_frequencies(*args)
    for trained, low, high in ((0, 1.0, 32.0), (4096, 32.0, 32.0), (4096, float("nan"), 1.0)):
        with pytest.raises(K.KnapError):
            K.knap_rope_frequencies(64, 1e4, K.KNAP_ROPE_PARTS, 2.0, trained, low, high)


@pytest.mark.gpu
def test_the_binding_refuses_what_the_library_cannot_see():
    import torch
    import paper_2508_06001_amd as K
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    freq = torch.ones((32,), dtype=torch.float64, device="cuda")
    pos = torch.zeros((4,), dtype=torch.int32, device="cuda")
    ok = dict(rot=64, layout=0, freq=freq, factor=1.0, positions=pos)
    K.knap_rope_fwd(x, x, q_out=torch.empty_like(x), k_out=torch.empty_like(x), **ok)
    for q, q_out, more in ((x.float(), x.float(), {}), (x, x[:3], {}), (x.transpose(1, 2).contiguous().transpose(1, 2), torch.empty_like(x), {}),
                           (x, torch.empty_like(x), dict(freq=freq.float())), (x, torch.empty_like(x), dict(freq=freq[:31])),
                           (x, torch.empty_like(x), dict(positions=pos.long())), (x, torch.empty_like(x), dict(positions=pos[:3])),
                           (x, torch.empty_like(x), dict(positions=None)), (x.cpu(), torch.empty_like(x), {}),
                           (x, torch.empty_like(x), dict(axis_pairs=[16, 16])), (x[0], torch.empty_like(x[0]), {}),
                           (x, torch.empty_like(x), dict(positions=pos.view(4, 1, 1).expand(4, 1, 2).contiguous()))):
        with pytest.raises(K.KnapError):
            K.knap_rope_fwd(q, None, q_out=q_out, k_out=None, **{**ok, **more})


def transposed(x, y, g, r, factor):
    """Rows in which <R x, g> = <x, R^T g> holds for y = R x and r = R^T g, each rounded to bf16.  A rounding moves a term by at most 2^-8 of it;
    taken as independent, of either sign, a sum of such terms leaves six times the root of their squares' sum with a probability of
    2 exp(-18).  Before the rounding a pair is off by 10^-6 of its two values (the head of this file), which the last term bounds for all."""
    a, b = y * g, x * r
    bar = 6 * 2.0 ** -8 * np.sqrt((a * a).sum(-1) + (b * b).sum(-1)) + 4e-6 * abs(factor) * np.sqrt((x * x).sum(-1) * (g * g).sum(-1))
    return np.abs(a.sum(-1) - b.sum(-1)) <= bar


FACTOR = 1.25


def wrong_backwards(x, g, pos, freq, rot, half):
    """Gradients as backwards would give them that are not the transpose."""
    turned = lambda sign, f=FACTOR: rope_ref(g, pos, freq, f, rot, half, sign)[0]  # noqa: E731
    rng = np.random.default_rng(12)
    return {"the forward's sign": turned(1.0), "not turned": g, "the factor alone": FACTOR * g, "without the factor": turned(-1.0, 1.0),
            "factor's inverse": turned(-1.0, 1.0 / FACTOR), "the other layout": rope_ref(g, pos, freq, FACTOR, rot, not half, -1.0)[0],
            "one position on": rope_ref(g, pos + 1, freq, FACTOR, rot, half, -1.0)[0], "nothing": 0 * g, "noise": rng.standard_normal(g.shape)}


@pytest.mark.parametrize("half", [True, False])
def test_what_the_transpose_check_catches(half):
    """The formula, rounded, passes in every row; a backward that is anything else fails in some."""
    import torch
    rng = np.random.default_rng(5)
    bf16 = lambda t: f64(torch.from_numpy(np.ascontiguousarray(t)).bfloat16())  # noqa: E731
    T, H, d, rot = 200, 4, 64, 48
    x, g = bf16(rng.standard_normal((T, H, d))), bf16(rng.standard_normal((T, H, d)))
    pos = np.repeat(np.concatenate([np.arange(77), np.arange(123)])[:, None], rot // 2, 1)
    freq = 10000.0 ** (-2.0 * np.arange(rot // 2) / rot)
    y = bf16(rope_ref(x, pos, freq, FACTOR, rot, half)[0])
    assert transposed(x, y, g, bf16(rope_ref(g, pos, freq, FACTOR, rot, half, -1.0)[0]), FACTOR).all()
    for name, r in wrong_backwards(x, g, pos, freq, rot, half).items():
        caught = 1.0 - transposed(x, y, g, bf16(r), FACTOR).mean()
        assert caught > 0.2, (name, caught)


@pytest.mark.gpu
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("T,H,Hk,d,rot,given", [(200, 4, 4, 128, 128, False), (200, 4, 2, 64, 48, False), (131, 3, 1, 64, 20, True), (97, 2, 2, 10, 6, True)])
def test_backward_is_the_transpose_in_every_row(T, H, Hk, d, rot, given, half):
    import torch
    import paper_2508_06001_amd as K
    say(f"[gpu] rope transpose T={T} H={H}/{Hk} d={d} rot={rot} given={given} half={half}")
    g = torch.Generator(device="cuda").manual_seed(T + rot)
    q, k, gq, gk = (torch.randn((T, h, d), generator=g, device="cuda").bfloat16() for h in (H, Hk, H, Hk))
    at = dict(positions=torch.randint(0, 5000, (T,), generator=g, device="cuda", dtype=torch.int32)) if given else dict(cu_seqlens=[0, 77, 77, T])
    rope = K.RotaryPositions(rot, K.KNAP_ROPE_HALF if half else K.KNAP_ROPE_INTERLEAVED, K.knap_rope_frequencies(rot)[0], FACTOR, **at)
    q_out, k_out, rq, rk = (torch.empty_like(t) for t in (q, k, q, k))
    rope.forward(q, k, q_out, k_out)
    rope.backward(gq, gk, rq, rk)
    torch.cuda.synchronize()
    for x, y, e, r in ((q, q_out, gq, rq), (k, k_out, gk, rk)):
        assert transposed(f64(x), f64(y), f64(e), f64(r), FACTOR).all()
