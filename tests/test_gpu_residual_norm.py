"""Residual norm against the oracle in 64 bits, at its bounds (oracle/residual_norm.py): widths of every form, odd ones, types, norms, strides,
sequences of no rows, of one and of many, padded bags, both directions; and refusals."""
import numpy as np
import pytest

from gpu_util import say
from oracle import residual_norm as R

HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
TYPES = [("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp32")]
WIDTHS = [1, 2, 7, 8, 63, 64, 120, 128, 129, 200, 256, 257, 512, 520, 768, 1000, 1003, 1024, 1025, 1032, 1536, 1537, 2048, 2056, 4096, 4099, 5000,
          8192, 8193, 8200, 12345, 16384]
BAGS = {"one": [23], "some": [3, 0, 7, 1, 0, 0, 12, 1], "ones": [1] * 9}
EPS = float(np.float32(1e-5))
ALPHA = 0.75


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def torch_type(name):
    import torch
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


class Frame:
    """A (rows, width) view into a tensor of NaN that is `pad` columns wider and has a row more on both sides."""

    def __init__(self, rows, width, dtype, pad, value=None):
        import torch
        self.shift = 8 if pad and pad % 8 == 0 else min(pad, 3)
        self.big = torch.full((rows + 2, width + pad), float("nan"), dtype=dtype, device="cuda")
        self.view = self.big[1:-1, self.shift:self.shift + width]
        if value is not None:
            self.view.copy_(value)

    def around_is_untouched(self):
        import torch
        inside = torch.zeros_like(self.big, dtype=torch.bool)
        inside[1:-1, self.shift:self.shift + self.view.shape[1]] = True
        return bool(torch.isnan(self.big[~inside]).all())


def make(lens, width, xt, bt, seed=0, f=True, mod=True, weights=True, mod_type="fp32", w_type="fp32", norm=R.LAYER, post=R.NONE, pad=0, spread=None):
    import torch
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + 7 * sum(lens) + width)
    rows, n = sum(lens), len(lens)
    new = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    raw = new(rows, width) * (0.5 + torch.rand((rows, 1), generator=g, device="cuda")) + new(rows, 1)
    if spread is not None:
        raw = spread(raw)
    c = {"rows": rows, "width": width, "lens": lens, "norm": norm, "post_norm": post, "xt": xt, "bt": bt, "pad": pad}
    c["cu"] = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    c["x"] = Frame(rows, width, torch_type(xt), pad, raw).view
    c["f"] = Frame(rows, width, torch_type(bt), pad, new(rows, width) * 1.5 + 0.2).view if f else None
    c["dx_out"] = Frame(rows, width, torch_type(xt), pad, new(rows, width)).view
    c["dy"] = Frame(rows, width, torch_type(bt), pad, new(rows, width)).view if norm != R.NONE else None
    chunks = (0.5 * new(n, 6 * width)).to(torch_type(mod_type))
    take = lambda i, there: chunks[:, i * width:(i + 1) * width] if there and mod else None  # noqa: E731
    c["gate"], c["scale"], c["shift"] = take(2, f), take(4, norm != R.NONE), take(3, norm != R.NONE)
    w = lambda there: (1 + 0.5 * new(width)).to(torch_type(w_type)) if there and weights else None  # noqa: E731
    c["weight"], c["post_weight"] = w(norm != R.NONE), w(f)
    return c


def call(c, backward=True, wants=("dx", "df", "dgate", "dscale", "dshift", "dweight", "dpost_weight"), dx_out=True):
    """Both directions through the binding; results by name, every frame checked."""
    import torch
    import paper_2508_06001_amd as K
    rows, width, n, f32 = c["rows"], c["width"], len(c["lens"]), torch.float32
    tx, tb = torch_type(c["xt"]), torch_type(c["bt"])
    frames = {}

    def out(name, there, dtype):
        if not there:
            return None
        frames[name] = Frame(rows, width, dtype, c["pad"])
        return frames[name].view

    has_f, has_y = c["f"] is not None, c["norm"] != R.NONE
    x_out, y = out("x_out", has_f, tx), out("y", has_y, tb)
    stats = torch.full((4, rows), float("nan"), device="cuda")
    same = dict(norm=c["norm"], post_norm=c["post_norm"], weight=c["weight"], post_weight=c["post_weight"], gate=c["gate"], scale=c["scale"],
                cu_seqlens=c["cu"], alpha=ALPHA)
    K.knap_residual_norm_fwd(c["x"], c["f"], x_out, y, shift=c["shift"], eps=EPS, stats=stats, **same)
    got = {"x_out": x_out, "y": y}
    names = (("mean", "rstd") if has_y else (None, None)) + (("post_mean", "post_rstd") if c["post_norm"] != R.NONE else (None, None))
    for i, name in enumerate(names):
        if name:
            got[name] = stats[i]
        else:
            assert bool(torch.isnan(stats[i]).all())
    if backward:
        dx, df = out("dx", "dx" in wants, tx), out("df", has_f and "df" in wants, tb)
        big = torch.full((3, n, 3 * width), float("nan"), device="cuda")      # gradients of the vectors as parts of wider rows
        vec = {name: big[i][:, width:2 * width] if there and name in wants else None
               for i, (name, there) in enumerate((("dgate", has_f), ("dscale", has_y), ("dshift", has_y)))}
        dw, dwp = (torch.full((width,), float("nan"), device="cuda") if there and name in wants else None
                   for name, there in (("dweight", has_y), ("dpost_weight", has_f)))
        ws = torch.full((max(256, K.knap_residual_norm_bwd_workspace_bytes(rows, width, n)) // 4,), float("nan"), device="cuda").view(torch.uint8)
        K.knap_residual_norm_bwd(c["x"], c["f"], stats, c["dx_out"] if dx_out else None, c["dy"], dx, df, dweight=dw, dpost_weight=dwp, workspace=ws,
                                 **vec, **same)
        got.update(dx=dx, df=df, dweight=dw, dpost_weight=dwp, **vec)
        for i, name in enumerate(("dgate", "dscale", "dshift")):
            assert bool(torch.isnan(big[i][:, :width]).all()) and bool(torch.isnan(big[i][:, 2 * width:]).all()), name
    torch.cuda.synchronize()
    for name, frame in frames.items():
        assert frame.around_is_untouched(), name
    return {k: v for k, v in got.items() if v is not None}


def check(c, got, dx_out=True):
    h = lambda t: None if t is None else f64(t)  # noqa: E731
    backward = "dx" in got
    val, bound = R.residual_norm(f64(c["x"]), h(c["f"]), f64(c["cu"]).astype(int), c["norm"], c["post_norm"], ALPHA, EPS,
                                 **{k: h(c[k]) for k in R.NAMES}, dx_out=h(c["dx_out"]) if backward and dx_out else None,
                                 dy=h(c["dy"]) if backward else None, half_x=HALF[c["xt"]], half_b=HALF[c["bt"]])
    for name, t in got.items():
        err = np.abs(f64(t) - val[name])
        assert np.all(err <= bound[name]), (name, float(np.nanmax(err - bound[name])))


@pytest.mark.gpu
@pytest.mark.parametrize("xt,bt", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_widths(width, xt, bt):
    for bag, norm, post in (("some", R.LAYER, R.RMS), ("one", R.RMS, R.NONE)):
        say(f"[gpu] residual norm width={width} {xt} {bt} {bag}")
        c = make(BAGS[bag], width, xt, bt, norm=norm, post=post, mod_type="bf16" if width % 3 == 0 else "fp32", w_type="bf16" if width % 5 == 0 else "fp32")
        check(c, call(c))


@pytest.mark.gpu
@pytest.mark.parametrize("norm", [R.NONE, R.RMS, R.LAYER])
@pytest.mark.parametrize("post", [R.NONE, R.RMS, R.LAYER])
@pytest.mark.parametrize("f,mod,weights", [(True, True, True), (True, False, True), (True, True, False), (True, False, False), (False, True, True), (False, False, False)])
def test_what_may_be_left_out(norm, post, f, mod, weights):
    if not f and (norm == R.NONE or post != R.NONE):
        pytest.skip("no such operator")
    for width, (xt, bt) in ((264, TYPES[0]), (1001, TYPES[1]), (1536, TYPES[2])):
        say(f"[gpu] residual norm {norm} {post} f={f} mod={mod} weights={weights} width={width}")
        c = make(BAGS["some"], width, xt, bt, f=f, mod=mod, weights=weights, norm=norm, post=post)
        check(c, call(c))
        if norm != R.NONE:
            check(c, call(c, dx_out=False), dx_out=False)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 63, 64, 65, 511, 513, 1025, 20011])
@pytest.mark.parametrize("width", [128, 264, 1096])
def test_rows_and_where_sequences_end(rows, width):
    rng = np.random.default_rng(rows)
    cuts = np.sort(rng.integers(0, rows + 1, size=min(rows, 70)))
    lens = np.diff(np.concatenate([[0], cuts, [rows]])).tolist()
    say(f"[gpu] residual norm rows={rows} width={width} sequences={len(lens)}")
    for bag in (lens, [rows]):
        c = make([int(v) for v in bag], width, "bf16", "bf16", norm=R.LAYER, post=R.RMS)
        check(c, call(c))


@pytest.mark.gpu
def test_as_many_sequences_as_there_may_be():
    import paper_2508_06001_amd as K
    rng = np.random.default_rng(8)
    lens = [int(v) for v in rng.integers(0, 4, size=K.KNAP_MAX_SEQS)]
    say("[gpu] residual norm, 2048 sequences")
    c = make(lens, 136, "bf16", "bf16", norm=R.RMS)
    check(c, call(c))


@pytest.mark.gpu
@pytest.mark.parametrize("xt,bt", TYPES)
@pytest.mark.parametrize("width,pad", [(128, 8), (128, 5), (1000, 1), (2048, 2048), (1536, 4)])
def test_strides(width, pad, xt, bt):
    say(f"[gpu] residual norm width={width} pad={pad}")
    c = make(BAGS["some"], width, xt, bt, pad=pad, norm=R.LAYER, post=R.LAYER)
    check(c, call(c))


@pytest.mark.gpu
@pytest.mark.parametrize("width", [128, 129, 1536, 4096])
def test_rows_far_from_zero(width):
    say(f"[gpu] residual norm far from zero width={width}")
    c = make([20, 13], width, "fp32", "fp32", norm=R.LAYER, post=R.NONE, spread=lambda t: 100.0 + t)
    check(c, call(c))


@pytest.mark.gpu
def test_wanted_or_not_every_result_has_the_same_bits():
    import torch
    c = make(BAGS["some"], 520, "bf16", "bf16", norm=R.LAYER, post=R.RMS)
    whole = call(c)
    for wants in (("dx",), ("df",), ("dgate", "dweight"), ("dshift",), ("dscale", "dpost_weight"), ()):
        some = call(c, wants=wants)
        for k, v in some.items():
            assert torch.equal(v, whole[k]), k


@pytest.mark.gpu
@pytest.mark.parametrize("width", [264, 1536, 1001])
def test_rows_behind_the_last_sequence_are_left(width):
    import torch
    import paper_2508_06001_amd as K
    rows, lens = 61, [9, 0, 22]
    say(f"[gpu] residual norm, padded bag width={width}")
    c = make([rows], width, "bf16", "bf16", norm=R.LAYER, post=R.RMS, mod=False)
    g = torch.Generator(device="cuda").manual_seed(1)
    vec = [0.5 * torch.randn((3, width), generator=g, device="cuda") for _ in range(3)]
    cu = torch.tensor([0, 9, 9, 31], dtype=torch.int32, device="cuda")
    n = K.ResidualNorm(rows, width, cu, K.KNAP_NORM_LAYER, c["weight"], K.KNAP_NORM_RMS, c["post_weight"], ALPHA, EPS)
    for t in (n.x_out, n.y, n.dx, n.df, n.stats):
        t.fill_(7.0)
    n.forward(c["x"], c["f"], *vec)
    n.backward(c["x"], c["f"], c["dx_out"], c["dy"], *vec)
    torch.cuda.synchronize()
    for t in (n.x_out[31:], n.y[31:], n.dx[31:], n.df[31:], n.stats[:, 31:]):
        assert bool((t == 7.0).all())
    d = {k: (v[:31] if k in ("x", "f", "dx_out", "dy") else v) for k, v in c.items()}
    d.update(lens=lens, cu=cu, rows=31, gate=vec[0], scale=vec[1], shift=vec[2])
    check(d, {"x_out": n.x_out[:31], "y": n.y[:31], "dx": n.dx[:31], "df": n.df[:31], "dgate": n.dgate, "dscale": n.dscale, "dshift": n.dshift,
              "dweight": n.dweight, "dpost_weight": n.dpost_weight})


@pytest.mark.gpu
def test_in_place_no_rows_and_a_gate_for_all():
    import torch
    import paper_2508_06001_amd as K
    c = make([5, 12], 520, "fp32", "bf16", norm=R.RMS, mod=False)
    one = torch.randn((1, 520), device="cuda").expand(2, 520)        # stride 0
    n = K.ResidualNorm(17, 520, c["cu"], K.KNAP_NORM_RMS, c["weight"], post_weight=c["post_weight"], alpha=ALPHA, eps=EPS,
                       x_type=torch.float32)
    x_out, y = (t.clone() for t in n.forward(c["x"], c["f"], gate=one))
    dx, df = (t.clone() for t in n.backward(c["x"], c["f"], c["dx_out"], c["dy"], gate=one))
    c["gate"] = one
    check(c, {"x_out": x_out, "y": y, "dx": dx, "df": df, "dgate": n.dgate, "dweight": n.dweight})
    dgate = n.dgate.clone()
    n.dx = c["dx_out"].clone()
    n.backward(c["x"], c["f"], n.dx, c["dy"], gate=one)
    assert torch.equal(n.dx, dx) and torch.equal(n.df, df) and torch.equal(n.dgate, dgate)
    n.x_out = c["x"].clone()
    n.forward(n.x_out, c["f"], gate=one)
    assert torch.equal(n.x_out, x_out) and torch.equal(n.y, y)
    e = K.ResidualNorm(0, 520, torch.zeros((3,), dtype=torch.int32), K.KNAP_NORM_RMS, c["weight"], alpha=ALPHA, x_type=torch.float32)
    for t in (e._dgate, e._dscale, e._dshift, e.dweight):
        t.fill_(7.0)
    e.forward(c["x"][:0], c["f"][:0], one, one, one)
    e.backward(c["x"][:0], c["f"][:0], None, c["dy"][:0], one, one)
    torch.cuda.synchronize()
    for t in (e.dgate, e.dscale, e.dshift, e.dweight):
        assert not bool(t.any())


@pytest.mark.gpu
def test_a_bag_of_no_sequences():
    """Rows, all of them padding: nothing is written but the sums over all rows, which are zeros; sums of no sequence need no launch."""
    import torch
    import paper_2508_06001_amd as K
    cu = torch.zeros((1,), dtype=torch.int32, device="cuda")
    x, y = torch.ones((5, 64), device="cuda"), torch.full((5, 64), 7.0, device="cuda")
    grad = torch.full((64,), 7.0, device="cuda")
    K.knap_residual_norm_fwd(x, None, None, y, cu_seqlens=cu)
    at = {n: t.data_ptr() for n, t in (("x", x), ("dy", y), ("dx", y), ("cu", cu), ("stats", y), ("g", grad))}
    args = dict(BWD, x=at["x"], xt=1, bt=1, xs=64, rows=5, f=0, fs=0, cu=at["cu"], n=0, gate=0, scale=0, wp=0, w=0, post=0, norm=2, stats=at["stats"], dxo=0,
                dy=at["x"], dx=at["dx"], df=0, dgate=0, dscale=at["g"], dshift=0, dw=0, dwp=0, ws=0, nbytes=0)
    assert K.lib.knap_residual_norm_bwd(*args.values(), 0) == K.KNAP_OK
    torch.cuda.synchronize()
    assert bool((y == 7.0).all()) and bool((grad == 7.0).all())
    assert K.lib.knap_residual_norm_bwd(*dict(args, dscale=0, dw=at["g"]).values(), 0) == K.KNAP_OK
    torch.cuda.synchronize()
    assert bool((y == 7.0).all()) and not bool(grad.any())


@pytest.mark.gpu
def test_a_bad_row_stays_in_its_row():
    import torch
    for width, post in ((128, R.NONE), (1536, R.RMS), (1001, R.LAYER)):
        c = make([10, 30], width, "bf16", "bf16", norm=R.LAYER, post=post)
        c["x"][7, 3], c["f"][20, 100], c["dy"][33, 5] = float("nan"), float("inf"), float("nan")
        got = call(c)
        rows = lambda *r: torch.tensor([i in r for i in range(40)], device="cuda")  # noqa: E731
        for k in ("dx", "df"):
            assert torch.equal(~torch.isfinite(got[k]).all(1), rows(7, 20, 33)), k
        assert torch.equal(~torch.isfinite(got["y"]).all(1), rows(7, 20))


@pytest.mark.gpu
def test_captured_calls_follow_their_inputs():
    import torch
    import paper_2508_06001_amd as K
    c = make([700, 1, 0, 300], 768, "bf16", "bf16", norm=R.LAYER, post=R.RMS)
    new = lambda: K.ResidualNorm(1001, 768, c["cu"], K.KNAP_NORM_LAYER, c["weight"], K.KNAP_NORM_RMS, c["post_weight"], ALPHA, EPS)  # noqa: E731
    a, b = new(), new()
    vec = (c["gate"], c["scale"], c["shift"])
    results = lambda n: [n.x_out, n.y, n.dx, n.df, n.dgate, n.dscale, n.dshift, n.dweight, n.dpost_weight]  # noqa: E731

    def both(n):
        n.forward(c["x"], c["f"], *vec)
        n.backward(c["x"], c["f"], c["dx_out"], c["dy"], *vec)

    both(a)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        both(b)
    for turn in range(4):
        c["f"].normal_()
        c["gate"].mul_(-1.1)
        c["cu"][1:4] -= 3          # the bag's boundaries are read on the device
        a.cu.copy_(c["cu"])
        b.cu.copy_(c["cu"])
        graph.replay()
        a.workspace.fill_(255)
        both(a)
        torch.cuda.synchronize()
        for s, t in zip(results(a), results(b)):
            assert torch.equal(s, t), turn


@pytest.mark.gpu
def test_on_another_stream_than_the_current_one():
    import torch
    import paper_2508_06001_amd as K
    c = make([300, 211], 1536, "bf16", "bf16", norm=R.RMS)
    n = K.ResidualNorm(511, 1536, c["cu"], K.KNAP_NORM_RMS, c["weight"], post_weight=c["post_weight"], alpha=ALPHA, eps=EPS)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    n.forward(c["x"], c["f"], c["gate"], c["scale"], c["shift"], stream=s)
    n.backward(c["x"], c["f"], c["dx_out"], c["dy"], c["gate"], c["scale"], stream=s)
    s.synchronize()
    check(c, {"x_out": n.x_out, "y": n.y, "dx": n.dx, "df": n.df, "dgate": n.dgate, "dscale": n.dscale, "dshift": n.dshift})


FWD = dict(x=256, xt=0, xs=64, rows=4, width=64, f=512, bt=0, fs=64, cu=64, n=2, gate=256, gs=64, scale=256, shift=256, ms=64, mt=1, wp=256, w=256, wt=1,
           post=1, norm=2, alpha=1.0, eps=1e-5, xo=4096, xos=64, y=8192, ys=64, stats=256)
BWD = dict(x=256, xt=0, xs=64, rows=4, width=64, f=512, bt=0, fs=64, cu=64, n=2, gate=256, gs=64, scale=256, ms=64, mt=1, wp=256, w=256, wt=1, post=1, norm=2,
           alpha=1.0, stats=256, dxo=1024, dxos=64, dy=2048, dys=64, dx=4096, dxs=64, df=8192, dfs=64, dgate=16384, dgs=64, dscale=32768, dshift=65536,
           dms=64, dw=256, dwp=512, ws=256, nbytes=1 << 20)


def test_bad_arguments_are_refused_without_touching_a_gpu():
    import paper_2508_06001_amd as K
    bad, inf, nan = K.KNAP_ERR_INVALID_ARG, float("inf"), float("nan")
    fwd = lambda **kw: K.lib.knap_residual_norm_fwd(*{**FWD, **kw}.values(), 0)  # noqa: E731
    bwd = lambda **kw: K.lib.knap_residual_norm_bwd(*{**BWD, **kw}.values(), 0)  # noqa: E731
    none = dict(x=0, f=0, xo=0, y=0)
    assert fwd(rows=0, **none) == K.KNAP_OK and fwd(n=0) == K.KNAP_OK
    assert bwd(rows=0, x=0, f=0, dgate=0, dscale=0, dshift=0, dw=0, dwp=0, ws=0) == K.KNAP_OK
    both = [dict(x=0), dict(xt=2), dict(bt=-1), dict(bt=1), dict(mt=2), dict(wt=3), dict(rows=-1), dict(rows=1 << 31), dict(width=0),
            dict(width=K.KNAP_LAYER_NORM_MAX_WIDTH + 1), dict(xs=63), dict(fs=0), dict(n=-1), dict(cu=0), dict(cu=66), dict(post=3), dict(post=-1),
            dict(norm=3), dict(norm=-1), dict(alpha=inf), dict(alpha=nan), dict(x=257), dict(f=513), dict(gate=258), dict(scale=257), dict(w=258), dict(wp=255),
            dict(gs=-1), dict(ms=-64), dict(f=256), dict(f=0), dict(norm=0)]
    for wrong in both:
        assert fwd(**wrong) == bad, wrong
        assert bwd(**wrong) == bad, wrong
    assert fwd(n=K.KNAP_MAX_SEQS + 1) == bwd(n=K.KNAP_MAX_SEQS + 1) == K.KNAP_ERR_TOO_MANY_SEQS
    for wrong in (dict(xo=0), dict(y=0), dict(y=256), dict(y=512), dict(y=4096), dict(xo=512), dict(xo=256, xos=72), dict(eps=-1.0), dict(eps=nan), dict(eps=inf),
                  dict(xos=8), dict(ys=63), dict(stats=255), dict(shift=258), dict(f=0, xo=0, gate=0, wp=0), dict(f=0, xo=0, gate=0, post=0),
                  dict(f=0, xo=0, wp=0, post=0), dict(f=0, gate=0, wp=0, post=0), dict(norm=0, y=0), dict(norm=0, w=0, scale=0, shift=0)):
        assert fwd(**wrong) == bad, wrong
    for wrong in (dict(dy=0), dict(stats=0), dict(stats=258), dict(dx=256), dict(dx=512), dict(dx=2048), dict(dx=8192), dict(dx=1024, dxs=72), dict(df=256),
                  dict(df=512), dict(df=2048), dict(df=1024), dict(dgate=16386), dict(dgate=32768), dict(dscale=65536), dict(dw=512), dict(dgs=63),
                  dict(dms=8), dict(ws=0), dict(ws=128), dict(dxs=63), dict(dfs=1), dict(dys=0), dict(dxos=12), dict(norm=0, w=0, scale=0),
                  dict(norm=0, w=0, scale=0, dy=0), dict(f=0, gate=0, wp=0, post=0), dict(f=0, gate=0, wp=0, post=0, df=0)):
        assert bwd(**wrong) == bad, wrong
    need = K.knap_residual_norm_bwd_workspace_bytes(4, 64, 2)
    assert need >= ((4 + 2) * 3 + 4 * 2) * 64 * 4 and bwd(nbytes=need - 1) == K.KNAP_ERR_WORKSPACE_TOO_SMALL
    assert K.knap_residual_norm_bwd_workspace_bytes(0, 64, 1) == 0


@pytest.mark.gpu
def test_the_binding_refuses_what_the_library_cannot_see():
    import torch
    import paper_2508_06001_amd as K
    c = make([4, 3], 64, "fp32", "bf16", norm=R.RMS)
    x_out, y, stats = torch.empty_like(c["x"]), torch.empty((7, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((4, 7), device="cuda")
    good = dict(x=c["x"], f=c["f"], x_out=x_out, y=y, norm=K.KNAP_NORM_RMS, weight=c["weight"], post_weight=c["post_weight"], gate=c["gate"], scale=c["scale"],
                shift=c["shift"], cu_seqlens=c["cu"], stats=stats)
    K.knap_residual_norm_fwd(**good)
    for wrong in (dict(f=c["f"][:6]), dict(f=c["f"].half()), dict(f=c["f"].t().contiguous().t()), dict(y=y.float()), dict(x_out=x_out.bfloat16()), dict(y=y[:, :63]),
                  dict(weight=c["weight"][:63]), dict(weight=c["weight"].bfloat16()), dict(gate=c["gate"][:1]), dict(gate=c["gate"].bfloat16()),
                  dict(scale=c["scale"][:, :63]), dict(shift=c["shift"].contiguous()), dict(cu_seqlens=c["cu"].long()), dict(cu_seqlens=c["cu"][:2]),
                  dict(stats=stats[:3]), dict(x=c["x"].cpu()), dict(gate=c["gate"].cpu())):
        with pytest.raises(K.KnapError):
            K.knap_residual_norm_fwd(**{**good, **wrong})
    grad = torch.empty((2, 64), device="cuda")
    ws = torch.empty((1 << 16,), dtype=torch.uint8, device="cuda")
    good = dict(x=c["x"], f=c["f"], stats=stats, dx_out=c["dx_out"], dy=c["dy"], dx=x_out, df=y, norm=K.KNAP_NORM_RMS, weight=c["weight"],
                post_weight=c["post_weight"], gate=c["gate"], scale=c["scale"], cu_seqlens=c["cu"], dgate=grad, workspace=ws)
    K.knap_residual_norm_bwd(**good)
    for wrong in (dict(dgate=grad[:1]), dict(dgate=grad.double()), dict(dgate=grad[:, :32]), dict(dx=y), dict(df=x_out), dict(dy=c["dy"].float()),
                  dict(dx_out=c["dx_out"].bfloat16()), dict(stats=None), dict(workspace=None), dict(workspace=ws[:256]), dict(dweight=grad[0][:63]),
                  dict(stats=stats[:, :6])):
        with pytest.raises(K.KnapError):
            K.knap_residual_norm_bwd(**{**good, **wrong})
