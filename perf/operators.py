"""The operators around and beside packed attention: differential attention, rotary positions, layer norm.

A case is a plain dict; ``op`` names the operator.

* ``diff``  differential attention over one packed bag: ``lens`` (text, comma separated), ``H`` heads of ``d`` columns, two maps of
            d / 2 each; ``train`` forward and backward, else the forward alone; ``causal`` the mask.
* ``rope``  rotary positions of q and k (``H`` and ``Hk`` heads of ``d``, the first ``rot`` columns rotated): ``layout`` "half" or
            "interleaved"; ``axes`` pairs of each axis (text) with positions given per token, or "" for the position in the own
            sequence of the bag ``lens``; ``fused``: q and k are slices of one (T, 3, H, d) tensor; ``far``: largest given position;
            ``bwd`` the backward, which rotates gradients back.
* ``norm``  layer norm of ``rows`` rows of ``width``; ``x`` and ``y`` their types; ``train`` forward and backward, else the forward alone.
"""
from __future__ import annotations

import math
import random
from typing import Dict, List

import torch

own = False

# text + image tokens, the mixed-resolution benchmark bag (31464 tokens); one GPU's post-switch share of an 8-GPU bag
MIXED_RES = "1406,4130,361,328,4079,2615,1407,1355,502,1306,4533,2686,367,1413,1141,1359,2476"
POST_ULYSSES = "131072,32768,8192,8192,8192,8192"
# rotary frequencies for a context eight times the one trained on, scaled by parts; and the plain ones
SCALED = {"base": 500000.0, "kind": "parts", "scale": 8.0, "trained": 8192, "low": 1.0, "high": 32.0}
PLAIN = {"base": 10000.0, "kind": "none", "scale": 1.0, "trained": 0, "low": 0.0, "high": 0.0}
EPS = 1e-5
MOST_SCORES = 2.3e9       # padded scores of a drawn bag, all heads: below the largest listed one's
MOST_ELEMENTS = 2.0e8     # of a drawn tensor


def listed() -> List[Dict]:
    return [
        # the smallest call: four short sequences of two 64-wide heads, one training step's layer
        {"name": "diff_tiny", "op": "diff", "lens": "37,128,200,311", "H": 2, "d": 64, "causal": False, "train": True},
        # sampling one 1024 x 1024 image, conditional and unconditional prompt in one bag: forward only
        {"name": "diff_image_pair", "op": "diff", "lens": "4173,4096", "H": 24, "d": 128, "causal": False, "train": False},
        # the mixed-resolution training bag, a quarter of the heads, causal
        {"name": "diff_mixed_causal", "op": "diff", "lens": MIXED_RES, "H": 6, "d": 128, "causal": True, "train": True},
        # one long sequence on one GPU of a sequence-parallel bag: three heads
        {"name": "diff_long", "op": "diff", "lens": "16384", "H": 3, "d": 128, "causal": False, "train": True},
        # next tokens of 16 sequences, far positions: where the launch is all there is
        {"name": "rope_next_tokens", "op": "rope", "lens": "16", "H": 24, "Hk": 24, "d": 128, "rot": 128, "layout": "half",
         "axes": "64", "fused": False, "far": 130000, "scaled": True, "bwd": False},
        # the mixed-resolution bag: (text, row, column) positions of q and k inside one projection's result
        {"name": "rope_mixed", "op": "rope", "lens": MIXED_RES, "H": 24, "Hk": 24, "d": 128, "rot": 128, "layout": "interleaved",
         "axes": "8,28,28", "fused": True, "far": 4096, "scaled": False, "bwd": False},
        # gradients of the post-switch bag: positions in the own sequence, half of each head rotated, scaled for long contexts
        {"name": "rope_long_bwd", "op": "rope", "lens": POST_ULYSSES, "H": 3, "Hk": 3, "d": 128, "rot": 64, "layout": "half",
         "axes": "", "fused": False, "far": 0, "scaled": True, "bwd": True},
        # heads of 64 with an odd part rotated: 10 pairs, which no 16-byte unit divides evenly
        {"name": "rope_part", "op": "rope", "lens": "4173,613,1024", "H": 12, "Hk": 4, "d": 64, "rot": 20, "layout": "half",
         "axes": "", "fused": False, "far": 0, "scaled": False, "bwd": False},
        # a few rows of a small model, forward
        {"name": "norm_few", "op": "norm", "rows": 37, "width": 768, "x": "bf16", "y": "bf16", "train": False},
        # the mixed-resolution bag's rows, training
        {"name": "norm_rows", "op": "norm", "rows": 31464, "width": 1536, "x": "bf16", "y": "bf16", "train": True},
        # every head's row behind attention of one image: 4292 tokens of 24 heads
        {"name": "norm_heads", "op": "norm", "rows": 4292 * 24, "width": 128, "x": "bf16", "y": "bf16", "train": True},
        # a residual stream kept in 32 bits, of an odd width
        {"name": "norm_odd", "op": "norm", "rows": 8191, "width": 4099, "x": "fp32", "y": "bf16", "train": True},
    ]


def _log_int(rng: random.Random, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _lens(case: Dict) -> List[int]:
    return [int(x) for x in case["lens"].split(",")]


def _text(lens) -> str:
    return ",".join(str(int(x)) for x in lens)


def _draw_lens(rng: random.Random, tokens: int) -> List[int]:
    family = rng.choice(("single", "equal", "ragged"))
    if family == "single":
        return [tokens]
    n = _log_int(rng, 1, 32)
    if family == "equal":
        return [max(1, tokens // n)] * n
    parts = [rng.uniform(0.2, 1.0) for _ in range(n)]
    return [max(1, int(tokens * p / sum(parts))) for p in parts]


def draw(rng: random.Random) -> Dict:
    op = rng.choice(("diff", "diff", "rope", "norm"))
    if op == "diff":
        while True:
            H, d = rng.choice(((24, 128), (12, 128), (6, 128), (3, 128), (48, 64), (12, 64), (2, 64)))
            lens = _draw_lens(rng, _log_int(rng, 300, 16384))
            if len(lens) * H * float(max(lens)) ** 2 <= 0.35 * MOST_SCORES:
                return {"op": op, "lens": _text(lens), "H": H, "d": d, "causal": rng.random() < 0.5, "train": rng.random() < 0.7}
    if op == "rope":
        while True:
            H, d = rng.choice(((24, 128), (12, 128), (3, 128), (48, 64), (12, 64)))
            lens = _draw_lens(rng, _log_int(rng, 1, 100000))
            if sum(lens) * H * d > 0.4 * MOST_ELEMENTS:
                continue
            Hk = H if rng.random() < 0.7 else max(1, H // 3)
            rot = rng.choice((d, d, d, d // 2, d // 4, 20))
            axes = rng.choice(("", "", _text([rot // 2]), _text([2, rot // 4 - 1, rot // 2 - rot // 4 - 1])))
            return {"op": op, "lens": _text(lens), "H": H, "Hk": Hk, "d": d, "rot": rot, "layout": rng.choice(("half", "interleaved")),
                    "axes": axes, "fused": Hk == H and rng.random() < 0.5, "far": _log_int(rng, 100, 1000000) if axes else 0,
                    "scaled": rng.random() < 0.5, "bwd": rng.random() < 0.5}
    while True:
        rows = _log_int(rng, 1, 100000)
        width = rng.choice((64, 128, 768, 1536, 2048, 4096, _log_int(rng, 33, 9000), _log_int(rng, 33, 9000)))
        if rows * width <= 0.3 * MOST_ELEMENTS:
            x = rng.choice(("bf16", "bf16", "fp32"))
            return {"op": op, "rows": rows, "width": width, "x": x, "y": "bf16" if x == "bf16" else rng.choice(("bf16", "fp32")),
                    "train": rng.random() < 0.7}


def _normal(gen: torch.Generator, shape, dtype=torch.bfloat16) -> torch.Tensor:
    return torch.randn(shape, generator=gen, dtype=dtype, device="cuda")


def _cu(lens) -> torch.Tensor:
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return torch.tensor(cu, dtype=torch.int32, device="cuda")


def _frequencies(case: Dict):
    """float64 frequencies of the rotated pairs (radians per position) and the factor of the rotated columns."""
    how = SCALED if case["scaled"] else PLAIN
    axes = [int(x) for x in case["axes"].split(",")] if case["axes"] else [case["rot"] // 2]
    freq = []
    for n in axes:
        for i in range(n):
            f = how["base"] ** (-i / n)
            if how["kind"] == "parts":      # as many turns in the trained length as decide between f and f / scale
                turns = how["trained"] * f / (2 * math.pi)
                keep = min(1.0, max(0.0, (turns - how["low"]) / (how["high"] - how["low"])))
                f = keep * f + (1 - keep) * f / how["scale"]
            freq.append(f)
    return torch.tensor(freq, dtype=torch.float64, device="cuda"), (0.1 * math.log(how["scale"]) + 1.0 if how["kind"] == "parts" else 1.0)


_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def prepare(case: Dict, seed: int) -> Dict:
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    state: Dict = {"case": case}
    if case["op"] == "diff":
        lens, H, d = _lens(case), case["H"], case["d"]
        T = sum(lens)
        state.update(cu=_cu(lens), T=T, scale=1.0 / math.sqrt(d // 2))
        for name in ("q", "k", "v") + (("dout",) if case["train"] else ()):
            state[name] = _normal(gen, (T, H, d))
        state["lam"] = 0.2 + 0.6 * torch.rand((H,), generator=gen, device="cuda")
        # rows of the padded form: token of (sequence, place), T (a row of zeros) where there is none
        longest = max(lens)
        place = torch.arange(longest, device="cuda")[None, :]
        n = torch.tensor(lens, device="cuda")[:, None]
        state["there"] = place < n
        state["index"] = torch.where(place < n, state["cu"][:-1, None].long() + place, torch.full_like(place, T))
        if own:
            import paper_2508_06001_amd as K
            state["attn"] = K.VarlenDiffAttention(state["cu"].cpu().numpy(), H, d, state["scale"], state["lam"], causal=case["causal"],
                                                  train=case["train"])
    elif case["op"] == "rope":
        lens, H, Hk, d = _lens(case), case["H"], case["Hk"], case["d"]
        T = sum(lens)
        if case["fused"]:
            qkv = _normal(gen, (T, 3, H, d))
            state.update(q=qkv[:, 0], k=qkv[:, 1])
        else:
            state.update(q=_normal(gen, (T, H, d)), k=_normal(gen, (T, Hk, d)))
        state["cu"] = _cu(lens)
        axes = [int(x) for x in case["axes"].split(",")] if case["axes"] else []
        state["axes"] = axes
        state["pos"] = torch.randint(0, case["far"] + 1, (T, len(axes)), generator=gen, dtype=torch.int32, device="cuda") if axes else None
        state["pair_axis"] = torch.tensor([a for a, n in enumerate(axes) for _ in range(n)], device="cuda") if axes else None
        state["freq"], state["factor"] = _frequencies(case)
        state["q_out"] = torch.empty((T, H, d), dtype=torch.bfloat16, device="cuda")
        state["k_out"] = torch.empty((T, Hk, d), dtype=torch.bfloat16, device="cuda")
    else:
        rows, width = case["rows"], case["width"]
        # activations: a mean and a spread of their own per row
        x = _normal(gen, (rows, width), torch.float32) * (0.5 + torch.rand((rows, 1), generator=gen, device="cuda"))
        x += 0.5 * torch.randn((rows, 1), generator=gen, device="cuda")
        state["x"] = x.to(_TYPES[case["x"]])
        state["w"] = 1.0 + 0.1 * torch.randn((width,), generator=gen, device="cuda")
        state["b"] = 0.1 * torch.randn((width,), generator=gen, device="cuda")
        if case["train"]:
            state["dy"] = _normal(gen, (rows, width), _TYPES[case["y"]])
        if own:
            import paper_2508_06001_amd as K
            state["norm"] = K.LayerNorm(rows, width, state["w"], state["b"], EPS, x_type=_TYPES[case["x"]], y_type=_TYPES[case["y"]],
                                        train=case["train"])
    return state


def _diff_plain(s: Dict) -> Dict:
    case, T, lam = s["case"], s["T"], s["lam"]
    H, half = case["H"], case["d"] // 2
    index, there = s["index"], s["there"]

    def padded(x):      # (sequences, heads, longest, d)
        rows = torch.cat([x.float(), torch.zeros_like(x[:1], dtype=torch.float32)])
        return rows[index].transpose(1, 2).contiguous()

    def packed(x):
        return x.transpose(1, 2)[there]

    q, k, v = padded(s["q"]), padded(s["k"]), padded(s["v"])
    hidden = ~there[:, None, None, :]
    if case["causal"]:
        place = torch.arange(index.shape[1], device=index.device)
        hidden = hidden | (place[None, :] > place[:, None])
    w = lam[None, :, None, None]

    def softmax(m):
        cols = slice(m * half, (m + 1) * half)
        x = torch.matmul(q[..., cols].contiguous(), k[..., cols].transpose(-1, -2).contiguous()).mul_(s["scale"])
        x.masked_fill_(hidden, -math.inf)
        top = x.amax(-1, keepdim=True)
        x.sub_(top).exp_()
        total = x.sum(-1, keepdim=True)
        return x.div_(total), (top + total.log())[..., 0]

    p1, lse1 = softmax(0)
    p2, lse2 = softmax(1)
    o2 = torch.matmul(p2, v)
    out = torch.matmul(p1, v) - w * o2
    lse = torch.stack([lse1, lse2]).transpose(1, 2)[:, :, there]
    if not case["train"]:
        return {"out": packed(out).bfloat16(), "lse": lse}
    do = padded(s["dout"])
    dlam = -(do * o2).sum((0, 2, 3))
    dv = torch.matmul((p1 - w * p2).transpose(-1, -2).contiguous(), do)
    dp = torch.matmul(do, v.transpose(-1, -2).contiguous())
    d1 = (p1 * dp).sum(-1, keepdim=True)
    d2 = (p2 * dp).sum(-1, keepdim=True)
    ds1 = (dp - d1).mul_(p1)
    ds2 = dp.sub_(d2).mul_(p2).mul_(-w)
    dq = torch.cat([torch.matmul(ds1, k[..., :half].contiguous()), torch.matmul(ds2, k[..., half:].contiguous())], -1)
    dk = torch.cat([torch.matmul(ds1.transpose(-1, -2).contiguous(), q[..., :half].contiguous()),
                    torch.matmul(ds2.transpose(-1, -2).contiguous(), q[..., half:].contiguous())], -1)
    return {"out": packed(out).bfloat16(), "out2": packed(o2).bfloat16(), "lse": lse, "dq": packed(dq * s["scale"]).bfloat16(),
            "dk": packed(dk * s["scale"]).bfloat16(), "dv": packed(dv).bfloat16(), "dlambda": dlam}


def _rope_plain(s: Dict) -> Dict:
    case, rot = s["case"], s["case"]["rot"]
    T = s["q"].shape[0]
    if s["pos"] is None:
        t = torch.arange(T, device=s["q"].device)
        pos = (t - s["cu"][torch.searchsorted(s["cu"], t, right=True) - 1])[:, None]
    else:
        pos = s["pos"][:, s["pair_axis"]]
    angle = pos.double() * s["freq"]
    c = (angle.cos() * s["factor"]).float()[:, None, :]
    sn = (angle.sin() * (-s["factor"] if case["bwd"] else s["factor"])).float()[:, None, :]

    def turned(x):
        x = x.float()
        y = x.clone()
        if case["layout"] == "half":
            a, b = x[..., : rot // 2], x[..., rot // 2: rot]
            y[..., : rot // 2] = a * c - b * sn
            y[..., rot // 2: rot] = a * sn + b * c
        else:
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
            y[..., 0:rot:2] = a * c - b * sn
            y[..., 1:rot:2] = a * sn + b * c
        return y.bfloat16()

    return {"q": turned(s["q"]), "k": turned(s["k"])}


def _norm_plain(s: Dict) -> Dict:
    case = s["case"]
    x = s["x"].float()
    mean = x.mean(-1, keepdim=True)
    xc = x - mean
    rstd = (xc.square().mean(-1, keepdim=True) + EPS).rsqrt()
    xh = xc * rstd
    y = (xh * s["w"] + s["b"]).to(_TYPES[case["y"]])
    if not case["train"]:
        return {"y": y}
    dy = s["dy"].float()
    g = dy * s["w"]
    dx = rstd * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    return {"y": y, "mean": mean[:, 0], "rstd": rstd[:, 0], "dx": dx.to(_TYPES[case["x"]]), "dw": (dy * xh).sum(0), "db": dy.sum(0)}


def run(state: Dict):
    case = state["case"]
    if not own:
        return {"diff": _diff_plain, "rope": _rope_plain, "norm": _norm_plain}[case["op"]](state)
    import paper_2508_06001_amd as K
    if case["op"] == "diff":
        attn = state["attn"]
        out, lse = attn.forward(state["q"], state["k"], state["v"])
        if not case["train"]:
            return {"out": out, "lse": lse}
        dq, dk, dv, dlam = attn.backward(state["q"], state["k"], state["v"], state["dout"])
        return {"out": out, "out2": attn.out2, "lse": lse, "dq": dq, "dk": dk, "dv": dv, "dlambda": dlam}
    if case["op"] == "rope":
        call = K.knap_rope_bwd if case["bwd"] else K.knap_rope_fwd
        call(state["q"], state["k"], case["rot"], K.KNAP_ROPE_HALF if case["layout"] == "half" else K.KNAP_ROPE_INTERLEAVED,
             state["freq"], state["factor"], state["q_out"], state["k_out"], positions=state["pos"], axis_pairs=state["axes"],
             cu_seqlens=None if state["axes"] else state["cu"])
        return {"q": state["q_out"], "k": state["k_out"]}
    norm = state["norm"]
    y = norm.forward(state["x"])
    if not case["train"]:
        return {"y": y}
    dx, dw, db = norm.backward(state["x"], state["dy"])
    return {"y": y, "mean": norm.mean, "rstd": norm.rstd, "dx": dx, "dw": dw, "db": db}


def work(case: Dict) -> Dict:
    if case["op"] == "diff":
        lens, H, d = _lens(case), case["H"], case["d"]
        pairs = sum(n * (n + 1) / 2.0 if case["causal"] else float(n) * n for n in lens)
        tensor, rows = 2 * sum(lens) * H * d, 4 * sum(lens) * H
        # in q, k, v (dout), out out (the second map's, dq, dk, dv); two log-sums a row; scores and two products, and five backward
        return {"bytes": (9 if case["train"] else 4) * tensor + 2 * rows, "flops": (16.0 if case["train"] else 6.0) * H * d * pairs}
    if case["op"] == "rope":
        T, heads = sum(_lens(case)), case["H"] + case["Hk"]
        given = 4 * T * len(case["axes"].split(",")) if case["axes"] else 4 * (len(_lens(case)) + 1)
        return {"bytes": 4 * T * heads * case["d"] + given, "flops": 3.0 * T * heads * case["rot"]}
    rows, width = case["rows"], case["width"]
    sx, sy = (2 if case[n] == "bf16" else 4 for n in ("x", "y"))
    n = rows * width
    if not case["train"]:
        return {"bytes": n * (sx + sy) + 8 * width, "flops": 8.0 * n}
    return {"bytes": n * (2 * sx + 2 * sy) + 16 * width + 8 * rows, "flops": 22.0 * n}


def _diff_exact(case: Dict, s: Dict):
    """One sequence and one head at a time, in 64 bits."""
    lens, H, d = _lens(case), case["H"], case["d"]
    if sum(float(n) ** 2 for n in lens) * H > 3.0e9:
        return None
    h2, T, train = d // 2, sum(lens), case["train"]
    new = lambda: torch.zeros((T, H, d), dtype=torch.float64, device="cuda")  # noqa: E731
    out, out2, dq, dk, dv = new(), new(), new(), new(), new()
    lse = torch.zeros((2, H, T), dtype=torch.float64, device="cuda")
    dlam = torch.zeros((H,), dtype=torch.float64, device="cuda")
    r0 = 0
    for n in lens:
        rows = slice(r0, r0 + n)
        r0 += n
        for h in range(H):
            lam = s["lam"][h].double()
            v = s["v"][rows, h].double()
            p, o, parts = [], [], []
            for m in (0, 1):
                qm, km = (s[x][rows, h, m * h2:(m + 1) * h2].double() for x in ("q", "k"))
                scores = (qm @ km.T) * s["scale"]
                if case["causal"]:
                    scores = scores + torch.full((n, n), -math.inf, dtype=torch.float64, device="cuda").triu(1)
                lse[m, h, rows] = torch.logsumexp(scores, 1)
                p.append(torch.exp(scores - lse[m, h, rows][:, None]))
                o.append(p[m] @ v)
                parts.append((qm, km))
            out[rows, h] = o[0] - lam * o[1]
            out2[rows, h] = o[1]
            if not train:
                continue
            do = s["dout"][rows, h].double()
            dp = do @ v.T
            dlam[h] -= (do * o[1]).sum()
            dv[rows, h] = (p[0] - lam * p[1]).T @ do
            for m, sign in ((0, 1.0), (1, -lam)):
                ds = sign * p[m] * (dp - (do * o[m]).sum(1, keepdim=True))
                dq[rows, h, m * h2:(m + 1) * h2] = s["scale"] * (ds @ parts[m][1])
                dk[rows, h, m * h2:(m + 1) * h2] = s["scale"] * (ds.T @ parts[m][0])
    if not train:
        return {"out": out, "lse": lse}
    return {"out": out, "out2": out2, "lse": lse, "dq": dq, "dk": dk, "dv": dv, "dlambda": dlam}


def _rope_exact(case: Dict, s: Dict) -> Dict:
    """Each pair as a complex number, turned."""
    lens, rot = _lens(case), case["rot"]
    if s["pos"] is None:
        own_pos = torch.cat([torch.arange(n, device="cuda") for n in lens])
        pos = own_pos[:, None].expand(-1, rot // 2)
    else:
        pos = torch.cat([s["pos"][:, a:a + 1].expand(-1, n) for a, n in enumerate(s["axes"])], 1)
    angle = pos.double() * s["freq"] * (-1.0 if case["bwd"] else 1.0)
    turn = torch.polar(torch.full_like(angle, s["factor"]), angle)[:, None, :]

    def of(x):
        x = x.double()
        head = x[..., :rot]
        if case["layout"] == "half":
            z = torch.complex(head[..., : rot // 2].contiguous(), head[..., rot // 2:].contiguous()) * turn
            head = torch.cat([z.real, z.imag], -1)
        else:
            z = torch.view_as_complex(head.reshape(*head.shape[:-1], rot // 2, 2).contiguous()) * turn
            head = torch.view_as_real(z).reshape(head.shape)
        return torch.cat([head, x[..., rot:]], -1)

    return {"q": of(s["q"]), "k": of(s["k"])}


def _norm_exact(case: Dict, s: Dict) -> Dict:
    x, w, b = s["x"].double(), s["w"].double(), s["b"].double()
    if case["train"]:
        x.requires_grad_(True)
        w.requires_grad_(True)
        b.requires_grad_(True)
    mean = x.sum(1) / case["width"]
    rstd = 1.0 / torch.sqrt(torch.var(x, 1, unbiased=False) + EPS)
    y = (x - mean[:, None]) * rstd[:, None] * w + b
    if not case["train"]:
        return {"y": y}
    dx, dw, db = torch.autograd.grad(y, (x, w, b), s["dy"].double())
    return {"y": y.detach(), "mean": mean.detach(), "rstd": rstd.detach(), "dx": dx, "dw": dw, "db": db}


def exact(case: Dict, seed: int):
    s = prepare(case, seed)
    return {"diff": _diff_exact, "rope": _rope_exact, "norm": _norm_exact}[case["op"]](case, s)
