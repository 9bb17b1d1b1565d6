"""Layer norm against the formula in 64 bits: widths of every form, odd ones, types, strides, few and many rows, both directions.

Bars.  Sums run in 32 bits over at most 32 values a thread, then over the threads (up to 9 steps in a tree of 512): each is off by less than
41 roundings of 2^-24 of the sum of magnitudes, below 2^-18.  With A = rstd max|x| of a row (xh and what the mean's error moves it by)
  y:  |w| (A 2^-17 + |xh| 2^-18) + |b| 2^-23 before its rounding,
  dx: rstd G (1 + A)^2 2^-16 with G = max |dy w| of the row (two means, each of products with an xh off by A 2^-17),
  dw: sum over rows |dy| (A 2^-17 + |xh| 2^-16) and db: sum |dy| 2^-16: a thread adds up rows one after the other, 512 of them at
      most here (101 roundings on the way through workgroups and their sums more),
and the rounding to the result's type, half a step of its value."""
import numpy as np
import pytest

from gpu_util import say

HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
TYPES = [("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp32")]
WIDTHS = [1, 2, 7, 8, 63, 64, 65, 120, 128, 129, 200, 256, 257, 511, 512, 520, 768, 1000, 1023, 1024, 1025, 1536, 2047, 2048, 2056, 2305, 4096,
          4099, 5000, 8192, 8193, 8200, 12345, 16384]


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def torch_type(name):
    import torch
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def norm_ref(x, w, b, eps):
    mean = x.mean(1)
    var = ((x - mean[:, None]) ** 2).mean(1)
    rstd = 1.0 / np.sqrt(var + eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    return mean, rstd, xh, xh * w + b


def norm_bwd_ref(xh, rstd, w, dy):
    g = dy * w
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def check_all(x, w, b, eps, dy, y, mean, rstd, dx, dw, db, x_type, y_type):
    m, r, xh, ref = norm_ref(x, w, b, eps)
    A = (r * np.abs(x).max(1))[:, None]
    off = np.abs(w) * (A * 2.0 ** -17 + np.abs(xh) * 2.0 ** -18) + np.abs(b) * 2.0 ** -23
    assert np.all(np.abs(y - ref) <= off + HALF[y_type] * (np.abs(ref) + off)), "y"
    assert np.all(np.abs(mean - m) <= 2.0 ** -18 * np.abs(x).mean(1) + 2.0 ** -24 * np.abs(m)), "mean"
    assert np.all(np.abs(rstd - r) <= 2.0 ** -16 * r * (1 + A[:, 0] * 2.0 ** -6)), "rstd"
    if dx is None:
        return
    gx, gw, gb = norm_bwd_ref(xh, r, w, dy)
    G = np.abs(dy * w).max(1, keepdims=True)
    off = r[:, None] * G * (1 + A) ** 2 * 2.0 ** -16
    assert np.all(np.abs(dx - gx) <= off + HALF[x_type] * (np.abs(gx) + off)), "dx"
    if dw is not None:
        assert np.all(np.abs(dw - gw) <= (np.abs(dy) * (A * 2.0 ** -17 + np.abs(xh) * 2.0 ** -16)).sum(0)), "dw"
    if db is not None:
        assert np.all(np.abs(db - gb) <= np.abs(dy).sum(0) * 2.0 ** -16), "db"


def run(rows, width, x_type, y_type, w_type="fp32", weights=True, pad=0, seed=0, spread=None):
    import torch
    import paper_2508_06001_amd as K
    g = torch.Generator(device="cuda").manual_seed(seed + 7 * rows + width)
    tx, ty = torch_type(x_type), torch_type(y_type)

    def place(t, dtype, shift):     # a (rows, width) view into NaN, `pad` columns wider, shifted by `shift` columns
        big = torch.full((rows + 2, width + pad), float("nan"), dtype=dtype, device="cuda")
        view = big[1:-1, shift:shift + width]
        if t is not None:
            view.copy_(t)
        return big, view

    raw = torch.randn((rows, width), generator=g, device="cuda") * (0.5 + torch.rand((rows, 1), generator=g, device="cuda"))
    raw += torch.randn((rows, 1), generator=g, device="cuda")
    if spread is not None:
        raw = spread(raw)
    shift = 8 if pad and pad % 8 == 0 else min(pad, 3)
    _, x = place(raw.to(tx), tx, shift)
    _, dy = place(torch.randn((rows, width), generator=g, device="cuda").to(ty), ty, shift)
    bigy, y = place(None, ty, shift)
    bigdx, dx = place(None, tx, shift)
    w = (1 + 0.5 * torch.randn((width,), generator=g, device="cuda")).to(torch_type(w_type)) if weights else None
    b = torch.randn((width,), generator=g, device="cuda").to(torch_type(w_type)) if weights else None
    mean, rstd = (torch.full((rows,), float("nan"), device="cuda") for _ in range(2))
    dw, db = (torch.full((width,), float("nan"), device="cuda") for _ in range(2))
    ws = torch.full((max(256, K.knap_layer_norm_bwd_workspace_bytes(rows, width)) // 4,), float("nan"), device="cuda").view(torch.uint8)
    eps = 1e-5
    K.knap_layer_norm_fwd(x, w, b, eps, y, mean, rstd)
    K.knap_layer_norm_bwd(x, w, mean, rstd, dy, dx, dw, db, ws)
    torch.cuda.synchronize()
    one, zero = np.ones(width), np.zeros(width)
    check_all(f64(x), one if w is None else f64(w), zero if b is None else f64(b), float(np.float32(eps)), f64(dy), f64(y), f64(mean), f64(rstd),
              f64(dx), f64(dw), f64(db), x_type, y_type)
    for big, view in ((bigy, y), (bigdx, dx)):      # nothing was written around the rows
        inside = torch.zeros_like(big, dtype=torch.bool)
        inside[1:-1, shift:shift + width] = True
        assert bool(torch.isnan(big[~inside]).all()) and bool(torch.isfinite(view).all())


@pytest.mark.gpu
@pytest.mark.parametrize("x_type,y_type", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_widths(width, x_type, y_type):
    say(f"[gpu] layer norm width={width} {x_type}->{y_type}")
    for rows in (1, 37):
        run(rows, width, x_type, y_type, w_type="bf16" if width % 3 == 0 else "fp32")


@pytest.mark.gpu
@pytest.mark.parametrize("x_type,y_type", TYPES)
@pytest.mark.parametrize("rows", [2, 3, 15, 16, 17, 63, 64, 65, 255, 1025, 20011])
@pytest.mark.parametrize("width", [128, 264])
def test_rows(rows, width, x_type, y_type):
    say(f"[gpu] layer norm rows={rows} width={width} {x_type}->{y_type}")
    run(rows, width, x_type, y_type)


@pytest.mark.gpu
@pytest.mark.parametrize("x_type,y_type", TYPES)
@pytest.mark.parametrize("width,pad", [(128, 8), (128, 5), (96, 160), (1000, 1), (2048, 2048), (4096, 16), (1536, 4)])
def test_strides_and_no_weights(width, pad, x_type, y_type):
    say(f"[gpu] layer norm width={width} pad={pad} {x_type}->{y_type}")
    run(50, width, x_type, y_type, pad=pad)
    run(50, width, x_type, y_type, pad=pad, weights=False)


@pytest.mark.gpu
@pytest.mark.parametrize("width", [128, 129, 1536, 4096])
def test_rows_far_from_zero_and_constant_rows(width):
    """A mean a hundred times the spread (x = 100 + noise in 32 bits), and rows whose values are all alike: rstd = 1 / sqrt(eps)."""
    say(f"[gpu] layer norm far from zero width={width}")
    run(33, width, "fp32", "fp32", spread=lambda t: 100.0 + t)
    import torch
    import paper_2508_06001_amd as K
    x = torch.full((5, width), 3.0, device="cuda")
    norm = K.LayerNorm(5, width, None, None, 1e-5, x_type=torch.float32, y_type=torch.float32)
    y = norm.forward(x)
    torch.cuda.synchronize()
    assert bool((y == 0).all()) and np.allclose(f64(norm.rstd), 1 / np.sqrt(np.float32(1e-5)), rtol=1e-6) and bool((norm.mean == 3.0).all())


@pytest.mark.gpu
def test_a_bad_row_stays_in_its_row():
    import torch
    import paper_2508_06001_amd as K
    x = torch.randn((40, 128), device="cuda").bfloat16()
    x[7, 3], x[20, 100] = float("nan"), float("inf")
    norm = K.LayerNorm(40, 128, torch.ones(128, device="cuda"), None)
    y = norm.forward(x)
    dx, dw, db = norm.backward(x, torch.ones_like(x))
    bad = torch.zeros((40,), dtype=torch.bool, device="cuda")
    bad[7] = bad[20] = True
    for t in (y, dx):
        assert torch.equal(~torch.isfinite(t).all(1), bad)
    assert db is None and bool(torch.isnan(dw).all())


@pytest.mark.gpu
def test_gradients_against_differences():
    """dx, dw, db of the kernels against central differences of the 64-bit formula: those of sum(y dy) at steps of 1e-5."""
    import torch
    import paper_2508_06001_amd as K
    rng = np.random.default_rng(4)
    rows, width = 3, 24
    x, dy = rng.standard_normal((2, rows, width)).astype(np.float32)
    w, b = rng.standard_normal((2, width)).astype(np.float32)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    norm = K.LayerNorm(rows, width, dev(w), dev(b), 1e-5, x_type=torch.float32, y_type=torch.float32)
    norm.forward(dev(x))
    got = [f64(t) for t in norm.backward(dev(x), dev(dy))]
    args = [x.astype(np.float64), w.astype(np.float64), b.astype(np.float64)]
    loss = lambda: (norm_ref(args[0], args[1], args[2], 1e-5)[3] * dy).sum()  # noqa: E731
    for a, grad in zip(args, got):
        for i in np.ndindex(a.shape):
            keep, h = a[i], 1e-5
            a[i] = keep + h
            up = loss()
            a[i] = keep - h
            diff = (up - loss()) / (2 * h)
            a[i] = keep
            assert abs(diff - grad[i]) <= 1e-4 * (1 + abs(diff)), (i, diff, grad[i])   # h^2 and 2^-52 / h are below 1e-6 here


@pytest.mark.gpu
def test_same_bits_no_rows_one_gradient_and_capture():
    import torch
    import paper_2508_06001_amd as K
    g = torch.Generator(device="cuda").manual_seed(2)
    x, dy = (torch.randn((3001, 768), generator=g, device="cuda").bfloat16() for _ in range(2))
    w, b = (torch.randn((768,), generator=g, device="cuda") for _ in range(2))
    norm = K.LayerNorm(3001, 768, w, b)
    norm.forward(x)
    first = [t.clone() for t in norm.backward(x, dy)]
    norm.workspace.fill_(255)
    again = norm.backward(x, dy)
    assert all(torch.equal(a, c) for a, c in zip(first, again))
    only = torch.empty((768,), device="cuda")        # one of the two sums, none of them
    dx = torch.empty_like(x)
    K.knap_layer_norm_bwd(x, w, norm.mean, norm.rstd, dy, dx, None, only, norm.workspace)
    assert torch.equal(only, first[2]) and torch.equal(dx, first[0])
    K.knap_layer_norm_bwd(x, w, norm.mean, norm.rstd, dy, dx.fill_(0), None, None, None)
    assert torch.equal(dx, first[0])
    empty = K.LayerNorm(0, 768, w, b)
    empty.forward(x[:0])
    _, dw, db = empty.backward(x[:0], dy[:0])
    assert bool((dw == 0).all()) and bool((db == 0).all())
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    other = K.LayerNorm(3001, 768, w, b)
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        other.forward(x)
        other.backward(x, dy)
    for turn in range(3):
        x.normal_(generator=g)
        graph.replay()
        y = norm.forward(x)
        grads = norm.backward(x, dy)
        torch.cuda.synchronize()
        assert torch.equal(y, other.y) and all(torch.equal(a, c) for a, c in zip(grads, (other.dx, other.dweight, other.dbias))), turn


def test_bad_arguments_are_refused_without_touching_a_gpu():
    import paper_2508_06001_amd as K
    bad = K.KNAP_ERR_INVALID_ARG

    def fwd(x=256, xt=0, xs=64, rows=4, width=64, w=256, b=256, wt=1, eps=1e-5, y=4096, yt=0, ys=64, mean=256, rstd=256):
        return K.lib.knap_layer_norm_fwd(x, xt, xs, rows, width, w, b, wt, eps, y, yt, ys, mean, rstd, 0)

    def bwd(x=256, xt=0, xs=64, rows=4, width=64, w=256, wt=1, mean=256, rstd=256, dy=512, yt=0, dys=64, dx=4096, dxs=64, dw=8192, db=16384,
            ws=256, n=1 << 20):
        return K.lib.knap_layer_norm_bwd(x, xt, xs, rows, width, w, wt, mean, rstd, dy, yt, dys, dx, dxs, dw, db, ws, n, 0)

    assert fwd(rows=0, x=0, y=0) == K.KNAP_OK and bwd(rows=0, x=0, dy=0, dx=0, dw=0, db=0, ws=0) == K.KNAP_OK
    for wrong in (dict(x=0), dict(y=0), dict(x=4096), dict(xt=2), dict(yt=-1), dict(yt=1), dict(wt=2), dict(rows=-1), dict(rows=1 << 31),
                  dict(width=0), dict(width=K.KNAP_LAYER_NORM_MAX_WIDTH + 1, xs=1 << 20, ys=1 << 20), dict(xs=63), dict(ys=0), dict(eps=-1.0),
                  dict(eps=float("nan")), dict(eps=float("inf")), dict(x=257), dict(xt=1, x=258), dict(w=258), dict(b=257), dict(mean=258), dict(rstd=254)):
        assert fwd(**wrong) == bad, wrong
    for wrong in (dict(x=0), dict(dy=0), dict(dx=0), dict(dx=256), dict(dx=512), dict(mean=0), dict(rstd=0), dict(ws=0), dict(ws=128), dict(dxs=63),
                  dict(dys=8), dict(dw=8194), dict(db=8192), dict(w=257), dict(wt=3), dict(rows=-1), dict(width=-5)):
        assert bwd(**wrong) == bad, wrong
    need = K.knap_layer_norm_bwd_workspace_bytes(4, 64)
    assert need >= 4 * 2 * 64 * 4 and bwd(n=need - 1) == K.KNAP_ERR_WORKSPACE_TOO_SMALL
    assert K.knap_layer_norm_bwd_workspace_bytes(0, 64) == 0 and K.knap_layer_norm_bwd_workspace_bytes(1 << 30, 64) == 1024 * 2 * 64 * 4


@pytest.mark.gpu
def test_the_binding_refuses_what_the_library_cannot_see():
    import torch
    import paper_2508_06001_amd as K
    x = torch.zeros((4, 64), device="cuda")
    w = torch.ones((64,), device="cuda")
    y = torch.empty_like(x)
    K.knap_layer_norm_fwd(x, w, w, 1e-5, y)
    for args in ((x.half(), w, w, y.half()), (x, w, w, y[:, :63]), (x, w[:63], w, y), (x, w, w.bfloat16(), y), (x.t(), w, w, y), (x.cpu(), w, w, y),
                 (x, w[::1].repeat(2)[::2], w, y)):
        with pytest.raises(K.KnapError):
            K.knap_layer_norm_fwd(args[0], args[1], args[2], 1e-5, args[3])
    with pytest.raises(K.KnapError):
        K.knap_layer_norm_fwd(x, w, w, 1e-5, y, mean=torch.empty((5,), device="cuda"))
