"""Differential attention against the 64-bit oracle: every element within what the roundings of its probabilities, score gradients and
outputs allow (oracle/diff_attention.py has the bounds), every output between NaN guard rows."""
import numpy as np
import pytest

from gpu_util import rel_fro, say
from oracle import diff_attention as D

GUARD = 64


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Run:
    """One forward and backward on guarded outputs that start as NaN."""

    def __init__(self, lens, H, d, causal, lam=None, seed=0, change=None, past=0, backward=True, scale=None):
        import torch
        import paper_2508_06001_amd as K
        self.cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        T = int(self.cu[-1])
        say(f"[gpu] diff n_seq={len(lens)} T={T} H={H} d={d} causal={causal} seed={seed} past={past}")
        g = torch.Generator(device="cuda").manual_seed(seed + T)
        self.x = {n: torch.randn((T + past, H, d), generator=g, device="cuda") for n in ("q", "k", "v", "dout")}
        if change:
            change(self.x)
        self.x = {n: t.bfloat16() for n, t in self.x.items()}
        self.lam = torch.tensor(np.linspace(-0.4, 1.3, H) if lam is None else lam, dtype=torch.float32, device="cuda")
        self.scale = float(np.float32((d // 2) ** -0.5 if scale is None else scale))
        self.big, self.y = {}, {}
        for n in ("out", "out2") + (("dq", "dk", "dv") if backward else ()):
            self.big[n] = torch.full((T + past + 2 * GUARD, H, d), float("nan"), dtype=torch.bfloat16, device="cuda")
            self.y[n] = self.big[n][GUARD:GUARD + T + past]
        self.big["lse"] = torch.full((2 * H * T + 2 * GUARD,), float("nan"), device="cuda")
        self.y["lse"] = self.big["lse"][GUARD:GUARD + 2 * H * T].view(2, H, T)
        self.T, self.H, self.d, self.causal, self.past = T, H, d, causal, past
        self.cu_dev = torch.from_numpy(self.cu).cuda()
        fwd, bwd = ((K.knap_varlen_diff_attn_causal_fwd, K.knap_varlen_diff_attn_causal_bwd) if causal
                    else (K.knap_varlen_diff_attn_fwd, K.knap_varlen_diff_attn_bwd))
        x, y, n = self.x, self.y, len(lens)
        fwd(x["q"], x["k"], x["v"], self.cu_dev, n, H, d, self.scale, self.lam, y["out"], y["out2"], y["lse"])
        if backward:
            nbytes = K.knap_varlen_diff_attn_bwd_workspace_bytes(T, n, H, d)
            ws = torch.full((max(nbytes, 256),), 255, dtype=torch.uint8, device="cuda")
            y["dlam"] = torch.full((H,), float("nan"), device="cuda")
            bwd(x["q"], x["k"], x["v"], self.cu_dev, n, H, d, self.scale, self.lam, y["out"], y["out2"], y["lse"], x["dout"], y["dq"], y["dk"], y["dv"],
                y["dlam"], T, ws)
        torch.cuda.synchronize()
        for name, big in self.big.items():      # nothing written around the rows of the bag, all of them written
            end = big.shape[0] - GUARD - (past if name != "lse" else 0)
            assert bool(torch.isnan(big[:GUARD]).all()) and bool(torch.isnan(big[end:]).all()), name
            assert bool(torch.isfinite(big[GUARD:end]).all()), name

    def check(self, heads=None, rel=None):
        heads = list(range(self.H)) if heads is None else heads
        x = {n: f64(t[:self.T, heads]) for n, t in self.x.items()}
        back = "dq" in self.y
        want, bound = D.diff_attn(x["q"], x["k"], x["v"], self.cu, f64(self.lam)[heads], self.scale, x["dout"] if back else None, self.causal)
        for n in want:
            got = f64(self.y[n][:, heads] if n == "lse" else self.y[n][heads] if n == "dlam" else self.y[n][:self.T, heads])
            err = np.abs(got - want[n])
            worst = float((err / (bound[n] + 1e-300)).max()) if err.size else 0.0
            say(f"[parity] {n}: worst share of its bound {worst:.3f}, rel {rel_fro(got, want[n]):.2e}")
            assert np.all(err <= bound[n]), (n, worst)
            if rel and n not in ("lse", "dlam"):
                assert rel_fro(got, want[n]) <= rel, n


BAGS = [[1], [2], [31], [32], [33], [63, 64, 65], [127, 128, 129], [37, 128, 200, 311], [0, 5, 0, 1, 300, 0], [257, 1, 255, 256], [700, 3]]


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", BAGS)
def test_ragged_bags(lens, d, causal):
    Run(lens, 3, d, causal).check()


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_many_sequences_and_many_heads(d, causal):
    rng = np.random.default_rng(6)
    Run([int(n) for n in rng.integers(0, 4, size=2048)], 2, d, causal).check()
    Run([5, 140, 90], 40, d, causal).check(heads=[0, 7, 39])
    Run([int(n) for n in rng.integers(100, 700, size=20)], 24, d, causal).check(heads=[11])


@pytest.mark.gpu
@pytest.mark.timeout(300)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_long_sequences(d, causal):
    """Three roundings of at most half a step each, of either sign: rms 2^-8 / sqrt(3) a rounding, 3.9e-3 together; the sums D_m from
    rounded outputs add less than another."""
    Run([4292, 130], 2, d, causal).check(heads=[1], rel=4.6e-3)


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_values_out_of_the_ordinary(d, causal):
    """Peaky keys, scores all far below zero with ragged ends, keys that rise along the sequence (the reference moves again and again), one map
    of zeros, and weights of the second map that are zero or negative."""
    def peaky(x):
        x["k"] *= 1 + 7 * (x["v"].abs() > 2.3)

    def below(x):
        x["q"][:] = 2.0
        x["k"][:] = -4.0 + 0.1 * x["k"]

    def rising(x):
        import torch
        x["k"] *= torch.linspace(0.1, 6.0, x["k"].shape[0], device="cuda")[:, None, None]

    def no_first(x):
        x["q"][..., : x["q"].shape[-1] // 2] = 0

    for change in (peaky, below, rising, no_first):
        Run([150, 70, 333], 2, d, causal, change=change, seed=3).check()
    Run([150, 70], 3, d, causal, lam=[0.0, -1.0, 2.5]).check()
    Run([150, 70], 2, d, causal, scale=1.0).check()


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_behind_the_last_sequence_and_other_sequences(d, causal):
    """A padded bag: rows behind the last sequence are left as they were.  NaN in one sequence and head stays there."""
    import torch
    run = Run([40, 200, 9], 2, d, causal, past=37)
    run.check()
    clean = {n: t.clone() for n, t in run.y.items()}

    def spoil(x):
        x["k"][100, 1, 3] = float("nan")
        x["v"][120, 1, 3] = float("inf")

    import paper_2508_06001_amd as K
    x = {n: t.clone() for n, t in run.x.items()}
    spoil(x)
    attn = K.VarlenDiffAttention(run.cu, 2, d, run.scale, run.lam, causal=causal)
    cut = {n: t[:249].contiguous() for n, t in x.items()}
    out, lse = attn.forward(cut["q"], cut["k"], cut["v"])
    dq, dk, dv, dlam = attn.backward(cut["q"], cut["k"], cut["v"], cut["dout"])
    torch.cuda.synchronize()
    for n, t in (("out", out), ("out2", attn.out2), ("dq", dq), ("dk", dk), ("dv", dv)):
        keep = torch.ones((249, 2), dtype=torch.bool, device="cuda")
        keep[40:240, 1] = False
        assert torch.equal(t[keep], clean[n][:249][keep]), n
    assert torch.equal(dlam[0], clean["dlam"][0]) and bool(torch.isnan(dlam[1]))


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_sequences_without_tokens_alone(d, causal):
    """The host cannot see that there are none: pointers are there, and what they point at stays as it was, but for dlambda."""
    import torch
    import paper_2508_06001_amd as K
    H, n = 3, 3
    say(f"[gpu] diff without tokens d={d} causal={causal}")
    rows = [torch.full((5, H, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(9)]
    lse, lam, dlam = torch.full((64,), float("nan"), device="cuda"), torch.ones((H,), device="cuda"), torch.full((H,), float("nan"), device="cuda")
    cu, ws = torch.zeros((n + 1,), dtype=torch.int32, device="cuda"), torch.zeros((256,), dtype=torch.uint8, device="cuda")
    fwd, bwd = ((K.knap_varlen_diff_attn_causal_fwd, K.knap_varlen_diff_attn_causal_bwd) if causal
                else (K.knap_varlen_diff_attn_fwd, K.knap_varlen_diff_attn_bwd))
    q, k, v, out, out2, dout, dq, dk, dv = rows
    fwd(q, k, v, cu, n, H, d, 0.1, lam, out, out2, lse)
    bwd(q, k, v, cu, n, H, d, 0.1, lam, out, out2, lse, dout, dq, dk, dv, dlam, 0, ws)
    torch.cuda.synchronize()
    assert not bool(dlam.any())
    assert all(bool(torch.isnan(t).all()) for t in rows + [lse])


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_bad_values_that_the_mask_hides(d):
    """NaN and infinities in rows 700 of k and v, 300 of q and dout, and -inf scores, reach at most 127 rows that do not see them."""
    import torch
    import paper_2508_06001_amd as K
    run = Run([1000], 2, d, True)
    x = {n: t.clone() for n, t in run.x.items()}
    attn = K.VarlenDiffAttention(run.cu, 2, d, run.scale, run.lam, causal=True)
    for row, names in ((700, ("k", "v")), (300, ("q", "dout"))):
        y = {n: t.clone() for n, t in x.items()}
        for n in names:
            y[n][row, 0, 1], y[n][row, 1, d - 1] = float("nan"), float("-inf")
        attn.forward(y["q"], y["k"], y["v"])
        attn.backward(y["q"], y["k"], y["v"], y["dout"])
        torch.cuda.synchronize()
        for n, t in (("out", attn.out), ("out2", attn.out2), ("dq", attn.dq), ("dk", attn.dk), ("dv", attn.dv)):
            if row == 700:        # queries before the key; their keys' gradients come from all queries behind them
                keep = slice(0, row - 127) if n in ("out", "out2", "dq") else None
            else:                 # the query's own rows, and gradients of the keys that it does not see
                keep = slice(row + 128, None)
            if keep is not None:
                assert torch.equal(t[keep], run.y[n][keep]), (row, n)


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
def test_same_bits_without_a_backward_captured_and_beside_each_other(causal):
    import torch
    import paper_2508_06001_amd as K
    lens, H, d = [300, 41, 800], 4, 128
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    T = int(cu[-1])
    g = torch.Generator(device="cuda").manual_seed(8)
    q, k, v, do = (torch.randn((T, H, d), generator=g, device="cuda").bfloat16() for _ in range(4))
    lam = torch.rand((H,), generator=g, device="cuda")
    new = lambda **kw: K.VarlenDiffAttention(cu, H, d, 0.125, lam, causal=causal, **kw)  # noqa: E731
    attn = new()

    def step(a):
        out, lse = a.forward(q, k, v)
        return [out, a.out2, lse, *a.backward(q, k, v, do)]

    first = [t.clone() for t in step(attn)]
    attn.workspace.fill_(170)
    again = step(attn)
    only, lse = new(train=False).forward(q, k, v)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again)) and torch.equal(only, first[0]) and torch.equal(lse, first[2])
    # two streams at once, a workspace each
    streams, twins = [torch.cuda.Stream() for _ in range(2)], [new() for _ in range(2)]
    for turn in range(3):
        for s, a in zip(streams, twins):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                step(a)
        torch.cuda.synchronize()
        for a in twins:
            assert all(torch.equal(x, y) for x, y in zip(first, (a.out, a.out2, a.lse, a.dq, a.dk, a.dv, a.dlam))), turn
    # captured, replayed with other values between eager calls
    graph, other = torch.cuda.CUDAGraph(), new()
    streams[0].wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=streams[0]):
        step(other)
    for turn in range(3):
        q.normal_(generator=g)
        lam.uniform_(generator=g)
        graph.replay()
        want = step(attn)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, (other.out, other.out2, other.lse, other.dq, other.dk, other.dv, other.dlam))), turn


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_more_items_than_workgroups_whatever_the_workspace_holds(d, causal):
    """Bags whose items are drawn from counters, by either kernel of the backward: the same bits whatever the workspace held, and right
    in a head that comes late in every list."""
    import torch
    import paper_2508_06001_amd as K
    run = Run([700, 130, 257, 512, 1, 333, 900, 64] * 4, 24, d, causal, seed=17)
    run.check(heads=[23])
    attn = K.VarlenDiffAttention(run.cu, 24, d, run.scale, run.lam, causal=causal)
    x = run.x
    for fill in (0, 1, 0x7f, 0xff):
        attn.workspace.fill_(fill)
        attn.forward(x["q"], x["k"], x["v"])
        got = dict(zip(("dq", "dk", "dv", "dlam"), attn.backward(x["q"], x["k"], x["v"], x["dout"])))
        torch.cuda.synchronize()
        for n, t in got.items():
            assert torch.equal(t, run.y[n][:run.T] if n != "dlam" else run.y[n]), (fill, n)


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_the_operators_together(d, causal):
    """A differential attention layer as a model has it: layer norm of the rows, rotary positions of both maps, the attention, layer norm of every
    head's row; the gradients go the way back.  Against the same chain in 64 bits.  Each of the up to six bf16 tensors on the way is rounded
    once, 2^-8 / sqrt(3) in the mean: 5.5e-3 of a result of one scale; normalising and differences of like terms take up to three times
    that, and no more than that is let pass."""
    import torch
    import paper_2508_06001_amd as K
    lens, H = [210, 1, 0, 333], 2
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    T = int(cu[-1])
    g = torch.Generator().manual_seed(21)
    x0, q, k, v, do = (torch.randn((T, H, d), generator=g).bfloat16() for _ in range(5))
    w, b = 1 + 0.2 * torch.randn((d,), generator=g), 0.2 * torch.randn((d,), generator=g)
    w1 = 1 + 0.2 * torch.randn((H * d,), generator=g)
    lam = torch.tensor([0.3, 0.7])
    scale = float(np.float32((d // 2) ** -0.5))
    freq, _ = K.knap_rope_frequencies(d // 2)
    dev = lambda t: t.cuda()  # noqa: E731
    rope = K.RotaryPositions(d // 2, K.KNAP_ROPE_HALF, freq, 1.0, cu_seqlens=cu)
    first = K.LayerNorm(T, H * d, dev(w1), None)
    attn = K.VarlenDiffAttention(cu, H, d, scale, dev(lam), causal=causal, rope=rope, norm=K.LayerNorm(T * H, d, dev(w), dev(b)))
    vn = first.forward(dev(x0).view(T, H * d)).view(T, H, d)                   # the values are the normalised rows themselves
    y, _ = attn.forward(dev(q), dev(k), vn)
    dq, dk, dvn, dlam = attn.backward(dev(q), dev(k), vn, dev(do))
    dx, dw1, _ = first.backward(dev(x0).view(T, H * d), dvn.view(T, H * d))
    torch.cuda.synchronize()

    leaves = {n: t.double().requires_grad_(True) for n, t in (("x", x0), ("q", q), ("k", k), ("w", w), ("b", b), ("w1", w1), ("lam", lam))}
    pos = torch.cat([torch.arange(n) for n in lens]).double()
    ang = pos[:, None, None, None] * torch.tensor(freq, dtype=torch.float64)

    def turned(t):
        t = t.view(T, H, 2, d // 2)
        a, c = t[..., : d // 4], t[..., d // 4:]
        return torch.cat([a * ang.cos() - c * ang.sin(), a * ang.sin() + c * ang.cos()], -1)

    def norm(t, weight, bias):
        m = t.mean(-1, keepdim=True)
        return (t - m) / ((t - m).square().mean(-1, keepdim=True) + 1e-5).sqrt() * weight + bias

    vals = norm(leaves["x"].reshape(T, H * d), leaves["w1"], 0.0).view(T, H, d)
    qt, kt = turned(leaves["q"]), turned(leaves["k"])
    outs = []
    for s in range(len(lens)):
        rows = slice(int(cu[s]), int(cu[s + 1]))
        n = lens[s]
        scores = torch.einsum("ihmc,jhmc->mhij", qt[rows], kt[rows]) * scale
        if causal:
            scores = scores.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), float("-inf"))
        p = scores.softmax(-1)
        outs.append(torch.einsum("hij,jhc->ihc", p[0] - leaves["lam"][:, None, None] * p[1], vals[rows]))
    ref = norm(torch.cat(outs), leaves["w"], leaves["b"])
    grads = dict(zip(leaves, torch.autograd.grad(ref, list(leaves.values()), do.double())))
    bar = 3 * 5.5e-3
    for name, got, want in (("y", y, ref), ("dq", dq, grads["q"]), ("dk", dk, grads["k"]), ("dx", dx.view(T, H, d), grads["x"]), ("dlam", dlam, grads["lam"]),
                            ("dw", attn.norm.dweight, grads["w"]), ("db", attn.norm.dbias, grads["b"]), ("dw1", dw1, grads["w1"])):
        rel = rel_fro(f64(got), want.detach().numpy())
        say(f"[parity] together d={d} causal={causal} {name} rel={rel:.2e}")
        assert rel <= bar, name


def test_bad_arguments_are_refused_without_touching_a_gpu():
    import paper_2508_06001_amd as K
    bad = K.KNAP_ERR_INVALID_ARG
    for f, g in ((K.lib.knap_varlen_diff_attn_fwd, K.lib.knap_varlen_diff_attn_bwd),
                 (K.lib.knap_varlen_diff_attn_causal_fwd, K.lib.knap_varlen_diff_attn_causal_bwd)):
        def fwd(q=256, k=512, v=768, cu=1024, n=1, H=2, d=64, scale=0.125, lam=64, out=2048, out2=4096, lse=8192):
            return f(q, k, v, cu, n, H, d, scale, lam, out, out2, lse, 0)

        def bwd(q=256, k=512, v=768, cu=1024, n=1, H=2, d=64, scale=0.125, lam=64, out=2048, out2=4096, lse=8192, do=16384, dq=256 * 65, dk=256 * 66,
                dv=256 * 67, dlam=256 * 68, T=100, ws=256 * 80, size=1 << 30):
            return g(q, k, v, cu, n, H, d, scale, lam, out, out2, lse, do, dq, dk, dv, dlam, T, ws, size, 0)

        assert fwd(n=0, q=0, k=0, v=0, cu=0, lam=0, out=0, out2=0, lse=0) == K.KNAP_OK
        assert bwd(n=0, q=0, k=0, v=0, cu=0, lam=0, out=0, out2=0, lse=0, do=0, dq=0, dk=0, dv=0, dlam=0, ws=0) == K.KNAP_OK
        common = [dict(q=0), dict(k=0), dict(v=0), dict(cu=0), dict(q=264), dict(cu=1026), dict(n=-1), dict(H=0), dict(d=96), dict(d=32), dict(scale=0.0),
                  dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(lam=0), dict(lam=66), dict(out=0), dict(out=2052),
                  dict(out2=4100), dict(lse=0), dict(lse=8194)]
        for wrong in common + [dict(out=256), dict(out=512), dict(out=768), dict(out2=2048), dict(out2=256)]:
            assert fwd(**wrong) == bad, wrong
        for wrong in common + [dict(out2=0), dict(do=0), dict(dq=0), dict(dk=0), dict(dv=0), dict(dlam=0), dict(dlam=2), dict(do=16388), dict(dq=256 * 66),
                               dict(dv=256 * 66), dict(dq=256), dict(dk=512), dict(dv=768), dict(dlam=64), dict(T=-1), dict(T=1 << 31), dict(ws=0), dict(ws=128)]:
            assert bwd(**wrong) == bad, wrong
        assert fwd(n=K.KNAP_MAX_SEQS + 1) == bwd(n=K.KNAP_MAX_SEQS + 1) == K.KNAP_ERR_TOO_MANY_SEQS
        need = K.knap_varlen_diff_attn_bwd_workspace_bytes(100, 1, 2, 64)
        assert need >= 5 * 100 * 2 * 4 and bwd(size=need - 1) == K.KNAP_ERR_WORKSPACE_TOO_SMALL
    assert K.knap_varlen_diff_attn_bwd_workspace_bytes(0, 1, 2, 64) == 0


@pytest.mark.gpu
def test_the_binding_refuses_what_the_library_cannot_see():
    import torch
    import paper_2508_06001_amd as K
    T, H, d = 8, 2, 64
    x = torch.zeros((T, H, d), dtype=torch.bfloat16, device="cuda")
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    lam, lse = torch.zeros((H,), device="cuda"), torch.zeros((2, H, T), device="cuda")
    call = lambda **kw: K.knap_varlen_diff_attn_fwd(**{**dict(q=x, k=x.clone(), v=x.clone(), cu_seqlens=cu, n_seq=1, H=H, d=d, scale=0.1, lam=lam,  # noqa: E731
                                                              out=torch.empty_like(x), out2=None, lse=lse), **kw})
    call()
    for wrong in (dict(q=x.float()), dict(k=x[:4]), dict(v=x.transpose(0, 1)), dict(lam=lam[:1]), dict(lam=lam.double()), dict(lse=lse.double()),
                  dict(out=x.cpu()), dict(lam=lam.cpu()), dict(cu_seqlens=cu.long()), dict(cu_seqlens=cu[:1]), dict(n_seq=2)):
        with pytest.raises(K.KnapError):
            call(**wrong)
