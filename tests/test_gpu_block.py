"""One transformer block over a packed bag as a training step runs it: norm and modulation, attention, gate, residual and the next norm, gated
feed-forward, the last residual; backward through all of it; and all gradients clipped by their global norm.  Against automatic differentiation of the
plain formulas in 64 bits.  The projections around attention are plain products in 32 bits, rounded to bf16.

Bars.  On its way from x to the block's output a value is rounded to bf16 some 12 times (norm, projection, probabilities, attention's output, projection,
residual, norm, a, b, h, y, residual), a gradient on its way back some 12 times more.  Each is off by up to 2^-8 of the value (0.42 of that as a rule), up or
down as its bits fall, and none of the block's steps (norms, softmax of scores below 4, products with weights of norm about 1, gates below 1) passes
an error on by more than twice its share.  So the 2-norm of a forward result's error is below 2 sqrt(12) 2^-8 of its own, that of a gradient's below 2 sqrt(24) 2^-8.
The residual stream is in 32 bits: its own error is the branches' share."""
import math

import numpy as np
import pytest

from gpu_util import say

FORWARD, BACKWARD = 2 * math.sqrt(12) * 2.0 ** -8, 2 * math.sqrt(24) * 2.0 ** -8
LENS, H, D_HEAD, HIDDEN, EPS, ALPHA = [37, 0, 150, 1, 90], 2, 64, 264, 1e-6, 0.75
WIDTH, ROWS = H * D_HEAD, sum(LENS)


def inputs():
    import torch
    g = torch.Generator(device="cuda").manual_seed(11)
    new = lambda *s, by=1.0: torch.randn(s, generator=g, device="cuda") * by  # noqa: E731
    p = {n: new(WIDTH, WIDTH, by=WIDTH ** -0.5).bfloat16() for n in ("wq", "wk", "wv", "wo")}
    p.update(wg=new(HIDDEN, WIDTH, by=WIDTH ** -0.5).bfloat16(), wu=new(HIDDEN, WIDTH, by=WIDTH ** -0.5).bfloat16(), wd=new(WIDTH, HIDDEN, by=HIDDEN ** -0.5).bfloat16())
    p.update(n1=1 + 0.2 * new(WIDTH), n2=1 + 0.2 * new(WIDTH), p1=1 + 0.2 * new(WIDTH))
    mod = 0.3 * new(len(LENS), 6 * WIDTH)
    return new(ROWS, WIDTH), p, mod, new(ROWS, WIDTH)


def plain(x, p, mod):
    import torch
    cu = np.concatenate([[0], np.cumsum(LENS)])
    m = [c.repeat_interleave(torch.tensor(LENS, device=x.device), 0) for c in mod.chunk(6, 1)]
    rms = lambda v: v / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)  # noqa: E731
    ln = lambda v: (v - v.mean(1, keepdim=True)) / torch.sqrt(v.var(1, unbiased=False, keepdim=True) + EPS)  # noqa: E731
    y = ln(x) * p["n1"] * (1 + m[1]) + m[0]
    q, k, v = ((y @ p[w].T).view(-1, H, D_HEAD) for w in ("wq", "wk", "wv"))
    o = []
    for a, b in zip(cu[:-1], cu[1:]):
        s = torch.einsum("ihd,jhd->hij", q[a:b], k[a:b]) / math.sqrt(D_HEAD)
        o.append(torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v[a:b]).reshape(b - a, WIDTH))
    f = torch.cat(o) @ p["wo"].T
    x1 = x + ALPHA * m[2] * (rms(f) * p["p1"])
    y = rms(x1) * p["n2"] * (1 + m[4]) + m[3]
    f = (torch.nn.functional.silu(y @ p["wg"].T) * (y @ p["wu"].T)) @ p["wd"].T
    return x1 + ALPHA * m[5] * f


def far(got, want):
    return float((got.double() - want).norm() / want.norm())


class Block:
    """The block with the framework's calls; gradients by name."""

    def __init__(self, p, mod):
        import torch
        import paper_2508_06001_amd as K
        cu = np.concatenate([[0], np.cumsum(LENS)]).astype(np.int32)
        f32 = torch.float32
        self.p, self.m = p, [c for c in mod.chunk(6, 1)]
        self.first = K.ResidualNorm(ROWS, WIDTH, cu, K.KNAP_NORM_LAYER, p["n1"], alpha=ALPHA, eps=EPS, x_type=f32, branch=False)
        self.attn = K.VarlenAttention(cu, H, D_HEAD, 1 / math.sqrt(D_HEAD))
        self.middle = K.ResidualNorm(ROWS, WIDTH, cu, K.KNAP_NORM_RMS, p["n2"], K.KNAP_NORM_RMS, p["p1"], ALPHA, EPS, x_type=f32)
        self.ffn = K.GatedFeedForward(ROWS, WIDTH, HIDDEN, p["wg"], p["wu"], p["wd"])
        self.last = K.ResidualNorm(ROWS, WIDTH, cu, K.KNAP_NORM_NONE, alpha=ALPHA, eps=EPS, x_type=f32)
        grads = [torch.zeros_like(p[n]) for n in ("wq", "wk", "wv", "wo")] + [self.ffn.dw_gate, self.ffn.dw_up, self.ffn.dw_down]
        grads += [self.first.dweight, self.middle.dweight, self.middle.dpost_weight]
        self.grads = dict(zip(("wq", "wk", "wv", "wo", "wg", "wu", "wd", "n1", "n2", "p1"), grads))
        self.clip = K.GradientClip(grads, 1.0)

    def product(self, a, w):
        return (a.float() @ w.float().T).bfloat16()

    def step(self, x, dout):
        import torch
        m, p = self.m, self.p
        _, y = self.first.forward(x, None, scale=m[1], shift=m[0])
        q, k, v = (self.product(y, p[w]).view(ROWS, H, D_HEAD) for w in ("wq", "wk", "wv"))
        o, _ = self.attn.forward(q, k, v)
        f1 = self.product(o.view(ROWS, WIDTH), p["wo"])
        x1, y2 = self.middle.forward(x, f1, m[2], m[4], m[3])
        f2 = self.ffn.forward(y2)
        out, _ = self.last.forward(x1, f2, m[5])
        # back
        dx1, df2 = self.last.backward(x1, f2, dout, None, m[5])
        dy2 = self.ffn.backward(y2, df2)[0]
        dx, df1 = self.middle.backward(x, f1, dx1, dy2, m[2], m[4])
        self.grads["wo"].copy_(df1.float().T @ o.view(ROWS, WIDTH).float())
        do = self.product(df1, p["wo"].T).view(ROWS, H, D_HEAD)
        dy = torch.zeros((ROWS, WIDTH), device="cuda")
        for w, g in zip(("wq", "wk", "wv"), self.attn.backward(q, k, v, do)):
            g = g.reshape(ROWS, WIDTH)
            self.grads[w].copy_(g.float().T @ y.float())
            dy += g.float() @ p[w].float()
        dx, _ = self.first.backward(x, None, dx, dy.bfloat16(), scale=m[1])
        dmod = torch.cat([self.first.dshift, self.first.dscale, self.middle.dgate, self.middle.dshift, self.middle.dscale, self.last.dgate], 1)
        return out, dx, dmod


@pytest.mark.gpu
def test_a_block_forward_backward_and_clipped():
    import torch
    say("[gpu] block")
    x, p, mod, dout = inputs()
    block = Block(p, mod)
    out, dx, dmod = block.step(x, dout)
    torch.cuda.synchronize()
    leaves = {n: t.double().requires_grad_(True) for n, t in dict(p, x=x, mod=mod).items()}
    want = plain(leaves["x"], {n: leaves[n] for n in p}, leaves["mod"])
    grads = dict(zip(leaves, torch.autograd.grad(want, list(leaves.values()), dout.double())))
    assert far(out, want.detach()) <= FORWARD
    assert far(dx, grads["x"]) <= BACKWARD
    assert far(dmod, grads["mod"]) <= BACKWARD
    assert not bool(dmod[1].any())              # the sequence without tokens
    for n, g in block.grads.items():
        assert far(g, grads[n]) <= BACKWARD, n
    before = {n: g.clone() for n, g in block.grads.items()}
    norm = float(block.clip.clip())
    torch.cuda.synchronize()
    total = math.sqrt(sum(float((g.double() ** 2).sum()) for g in before.values()))
    assert abs(norm - total) <= 2.0 ** -23 * total and norm > 1.0
    for n, g in block.grads.items():
        ref = before[n].double() / (total + 1e-6)
        assert bool(((g.double() - ref).abs() <= (2.0 ** -22 + (2.0 ** -8 if g.dtype is torch.bfloat16 else 2.0 ** -24)) * ref.abs() + 2.0 ** -133).all()), n


@pytest.mark.gpu
def test_a_captured_block_follows_its_inputs():
    """The whole step in a graph, products around attention and clipping with it, against the eager step."""
    import torch
    say("[gpu] block, captured")
    x, p, mod, dout = inputs()
    eager, held = Block(p, mod), Block(p, mod)

    def step(b):
        out = b.step(x, dout)
        b.clip.clip()
        return out

    step(eager)
    step(held)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        got = step(held)
    for turn in range(3):
        x.normal_()
        mod.mul_(-0.9)
        graph.replay()
        want = step(eager)
        torch.cuda.synchronize()
        for a, b in zip(list(got) + list(held.grads.values()), list(want) + list(eager.grads.values())):
            assert torch.equal(a, b), turn
