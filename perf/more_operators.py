"""The rest of a transformer block around packed attention, and the end of a training step.

A case is a plain dict; ``op`` names the operator.

* ``norm``  the norm behind a branch, its gate and residual scale, and the norm and modulation in front of the next branch, over the rows of a
            packed bag: ``lens`` (text, comma separated), ``width``; ``x`` the type of the residual stream, ``branch`` that of the branch's
            output and of the next one's input; ``post`` and ``pre`` "none", "rms" or "layer"; ``f``: there is a branch; ``modulated``: gate,
            scale and shift per sequence; ``weights``: learned weights in both norms; ``train`` forward and backward, else the forward alone.
* ``ffn``   gated feed-forward of ``tokens`` rows, ``width`` and ``hidden`` columns, ``act`` "silu" or "gelu" (the tanh form); ``train`` as
            above.
* ``clip``  the global norm of many gradients and clipping by it: ``sizes`` (text: "count x elements" of groups of tensors), ``type`` "bf16", "fp32"
            or "mixed"; ``bite``: the norm over the largest norm allowed.
"""
from __future__ import annotations

import math
import random
from typing import Dict, List

import torch

own = False

# text + image tokens, the mixed-resolution benchmark bag (31464 tokens); one GPU's share of an 8-GPU bag
MIXED_RES = "1406,4130,361,328,4079,2615,1407,1355,502,1306,4533,2686,367,1413,1141,1359,2476"
LONG_SHARE = "16384,4096,1024,1024,1024,1024"
EPS = 1e-6
CLIP_EPS = 1e-6
ALPHA = 0.75                 # the residual scale of the cases
MOST_ELEMENTS = 3.5e7        # rows times width of a drawn norm
MOST_PRODUCTS = 1.9e11       # tokens times width times hidden of a drawn feed-forward
MOST_GRADIENTS = 1.6e8       # elements of a drawn list


def listed() -> List[Dict]:
    return [
        # the next step of five short samples of a small model, forward: where the launch is all there is
        {"name": "norm_few", "op": "norm", "lens": "1,1,1,1,1", "width": 768, "x": "bf16", "branch": "bf16", "post": "none", "pre": "rms", "f": True,
         "modulated": True, "weights": True, "train": False},
        # the mixed-resolution bag, modulated by each sample's own vectors, training
        {"name": "norm_mixed", "op": "norm", "lens": MIXED_RES, "width": 1536, "x": "bf16", "branch": "bf16", "post": "none", "pre": "layer",
         "f": True, "modulated": True, "weights": False, "train": True},
        # norms on both sides of the branch, a residual stream kept in 32 bits, one long sequence and some short ones
        {"name": "norm_both_sides", "op": "norm", "lens": LONG_SHARE, "width": 2048, "x": "fp32", "branch": "bf16", "post": "rms", "pre": "rms",
         "f": True, "modulated": True, "weights": True, "train": True},
        # an odd width, empty sequences among the others, norms of both kinds
        {"name": "norm_odd", "op": "norm", "lens": "1201,0,37,3001,0,0,1,2503,777,64", "width": 1003, "x": "fp32", "branch": "fp32", "post": "layer",
         "pre": "rms", "f": True, "modulated": True, "weights": True, "train": True},
        # one token: the weights are read, and that is all
        {"name": "ffn_token", "op": "ffn", "tokens": 1, "width": 2048, "hidden": 5504, "act": "silu", "train": False},
        # the next tokens of 24 samples of a wider model
        {"name": "ffn_next_tokens", "op": "ffn", "tokens": 24, "width": 4096, "hidden": 10944, "act": "silu", "train": False},
        # sampling one 1024 x 1024 image with its prompt: forward
        {"name": "ffn_image", "op": "ffn", "tokens": 4173, "width": 2048, "hidden": 5504, "act": "gelu", "train": False},
        # the mixed-resolution bag, training
        {"name": "ffn_mixed", "op": "ffn", "tokens": 31464, "width": 1536, "hidden": 4096, "act": "silu", "train": True},
        # a short bag of a narrow model, sizes that no tile divides
        {"name": "ffn_ragged", "op": "ffn", "tokens": 613, "width": 1000, "hidden": 2664, "act": "gelu", "train": True},
        # a small model's gradients: 38 tensors, none of them large
        {"name": "clip_small", "op": "clip", "sizes": "12x768,12x589824,12x1179,2x98304", "type": "bf16", "bite": 3.0},
        # one GPU's share of a model of many blocks: matrices and vectors of 16 blocks
        {"name": "clip_blocks", "op": "clip", "sizes": "48x6291456,32x1536,16x2359296", "type": "bf16", "bite": 20.0},
        # gradients in 32 bits with vectors between them, sizes that no 16-byte unit divides; below the limit, so that nothing shrinks
        {"name": "clip_odd", "op": "clip", "sizes": "7x4194301,300x1003,5x999983,40x1", "type": "mixed", "bite": 0.5},
    ]


def _log_int(rng: random.Random, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _lens(case: Dict) -> List[int]:
    return [int(x) for x in case["lens"].split(",")]


def _draw_lens(rng: random.Random, tokens: int) -> List[int]:
    n = min(tokens, _log_int(rng, 1, 64))
    if rng.random() < 0.3:
        return [max(1, tokens // n)] * n
    parts = [rng.choice((0.0, 1.0, 1.0, 1.0)) * rng.uniform(0.1, 1.0) for _ in range(n)]
    total = sum(parts)
    return [int(tokens * p / total) for p in parts] if total > 0 else [tokens]


def draw(rng: random.Random) -> Dict:
    op = rng.choice(("norm", "norm", "ffn", "ffn", "clip"))
    if op == "norm":
        while True:
            width = rng.choice((128, 768, 1536, 2048, 4096, _log_int(rng, 33, 9000), 8 * _log_int(rng, 8, 1200)))
            lens = _draw_lens(rng, _log_int(rng, 1, 60000))
            if sum(lens) * width > MOST_ELEMENTS or sum(lens) == 0:
                continue
            x = rng.choice(("bf16", "bf16", "fp32"))
            f = rng.random() < 0.85
            return {"op": op, "lens": ",".join(str(n) for n in lens), "width": width, "x": x,
                    "branch": "bf16" if x == "bf16" else rng.choice(("bf16", "bf16", "fp32")), "post": rng.choice(("none", "none", "rms", "layer")) if f else "none",
                    "pre": rng.choice(("rms", "layer", "none")) if f else rng.choice(("rms", "layer")), "f": f, "modulated": rng.random() < 0.75,
                    "weights": rng.random() < 0.5, "train": rng.random() < 0.7}
    if op == "ffn":
        while True:
            tokens = _log_int(rng, 1, 40000)
            width = rng.choice((768, 1536, 2048, 8 * _log_int(rng, 8, 512), 8 * _log_int(rng, 8, 512)))
            hidden = rng.choice((64 * -(-width // 24), 4 * width, 8 * _log_int(rng, 8, 1400)))
            if tokens * width * hidden <= MOST_PRODUCTS and width * hidden <= 5e7:
                return {"op": op, "tokens": tokens, "width": width, "hidden": hidden, "act": rng.choice(("silu", "gelu")), "train": rng.random() < 0.6}
    while True:
        groups = [(_log_int(rng, 1, 200), _log_int(rng, 1, 8000000)) for _ in range(rng.randint(1, 5))]
        if sum(n * m for n, m in groups) <= MOST_GRADIENTS:
            return {"op": op, "sizes": ",".join(f"{n}x{m}" for n, m in groups), "type": rng.choice(("bf16", "bf16", "fp32", "mixed")),
                    "bite": rng.choice((0.5, 3.0, 50.0))}


_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _normal(gen: torch.Generator, shape, dtype=torch.float32) -> torch.Tensor:
    return torch.randn(shape, generator=gen, dtype=dtype, device="cuda")


def _sizes(case: Dict) -> List[int]:
    """Elements of each tensor of the list."""
    return [int(m) for n, m in (g.split("x") for g in case["sizes"].split(",")) for _ in range(int(n))]


def _buckets(tensors):
    """One buffer of zeros for each type and every tensor's part of it."""
    total, start = {}, []
    for g in tensors:
        start.append(total.get(g.dtype, 0))
        total[g.dtype] = start[-1] + -(-g.numel() // 64) * 64
    flat = {t: torch.zeros((n,), dtype=t, device="cuda") for t, n in total.items()}
    return flat, [flat[g.dtype][at:at + g.numel()] for g, at in zip(tensors, start)]


def prepare(case: Dict, seed: int) -> Dict:
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s: Dict = {"case": case}
    if own:
        import paper_2508_06001_amd as K
    if case["op"] == "norm":
        lens, width = _lens(case), case["width"]
        rows, n = sum(lens), len(lens)
        tx, tb = _TYPES[case["x"]], _TYPES[case["branch"]]
        cu = [0]
        for m in lens:
            cu.append(cu[-1] + m)
        s["cu"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
        # the residual stream: rows of their own size and mean, a few columns much larger than the rest
        x = _normal(gen, (rows, width)) * (0.5 + 2.0 * torch.rand((rows, 1), generator=gen, device="cuda")) + 0.3 * _normal(gen, (rows, 1))
        x[:, :: max(1, width // 3)] *= 8.0
        s["x"] = x.to(tx)
        s["f"] = (_normal(gen, (rows, width)) * 1.5 + 0.1).to(tb) if case["f"] else None
        s["gate"] = s["scale"] = s["shift"] = s["w"] = s["wp"] = None
        if case["modulated"]:       # chunks of one projection of every sample's conditioning
            mod = 0.4 * _normal(gen, (n, 6 * width))
            s["gate"], s["scale"], s["shift"] = (mod[:, i * width:(i + 1) * width] for i in (2, 4, 3))
        if case["weights"]:
            s["w"] = 1.0 + 0.2 * _normal(gen, (width,))
            s["wp"] = 1.0 + 0.2 * _normal(gen, (width,))
        if not case["f"] or case["post"] == "none":
            s["wp"] = None
        if not case["f"]:
            s["gate"] = None
        if case["pre"] == "none":
            s["w"] = s["scale"] = s["shift"] = None
        if case["train"]:
            s["dx_out"] = _normal(gen, (rows, width)).to(tx)
            s["dy"] = _normal(gen, (rows, width)).to(tb) if case["pre"] != "none" else None
        if own:
            kinds = {"none": K.KNAP_NORM_NONE, "rms": K.KNAP_NORM_RMS, "layer": K.KNAP_NORM_LAYER}
            s["op"] = K.ResidualNorm(rows, width, s["cu"], norm=kinds[case["pre"]], weight=s["w"], post_norm=kinds[case["post"]],
                                     post_weight=s["wp"], alpha=ALPHA, eps=EPS, x_type=tx, branch_type=tb, branch=case["f"], train=case["train"])
    elif case["op"] == "ffn":
        T, D, F = case["tokens"], case["width"], case["hidden"]
        bf16 = torch.bfloat16
        s["x"] = _normal(gen, (T, D)).to(bf16)
        s["wg"] = (_normal(gen, (F, D)) / math.sqrt(D)).to(bf16)
        s["wu"] = (_normal(gen, (F, D)) / math.sqrt(D)).to(bf16)
        s["wd"] = (_normal(gen, (D, F)) / math.sqrt(F)).to(bf16)
        if case["train"]:
            s["dy"] = _normal(gen, (T, D)).to(bf16)
        if own:
            s["op"] = K.GatedFeedForward(T, D, F, s["wg"], s["wu"], s["wd"], K.KNAP_SILU if case["act"] == "silu" else K.KNAP_GELU_TANH,
                                         train=case["train"])
    else:
        sizes = _sizes(case)
        s["grads"] = []
        for i, n in enumerate(sizes):
            t = torch.float32 if case["type"] == "fp32" or (case["type"] == "mixed" and i % 3) else torch.bfloat16
            s["grads"].append((_normal(gen, (n,)) * (10.0 ** ((i % 7) - 5))).to(t))
        # the norm that these have on the average, over the bite
        s["max_norm"] = math.sqrt(sum(n * 100.0 ** ((i % 7) - 5) for i, n in enumerate(sizes))) / case["bite"]
        # where the optimizer takes them from: one buffer for each type, in which every tensor starts on 64 elements
        s["flat"], s["out"] = _buckets(s["grads"])
        if own:
            s["op"] = K.GradientClip(s["grads"], s["max_norm"], eps=CLIP_EPS, out=s["out"])
    return s


def _rows_of(s: Dict):
    """The sequence of every row."""
    t = torch.arange(s["x"].shape[0], dtype=torch.int32, device=s["x"].device)
    return torch.searchsorted(s["cu"], t, right=True) - 1


def _normed(x, kind: str):
    """(x - mean) rstd and rstd."""
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    return x * r, r


def _normed_back(g, xh, r, kind: str):
    out = g - xh * (g * xh).mean(-1, keepdim=True)
    if kind == "layer":
        out = out - g.mean(-1, keepdim=True)
    return out * r


def _norm_plain(s: Dict) -> Dict:
    case = s["case"]
    seq, lens = _rows_of(s), _lens(case)
    tx, tb = _TYPES[case["x"]], _TYPES[case["branch"]]

    def per_row(v, none):
        return none if v is None else v.float()[seq]

    def over_rows(v):       # sums of each sequence's rows
        return torch.stack([part.sum(0, dtype=torch.float64) for part in torch.split(v, lens)])

    out = {}
    x = s["x"].float()
    gate, scale = per_row(s["gate"], 1.0), per_row(s["scale"], 0.0)
    w = 1.0 if s["w"] is None else s["w"]
    wp = 1.0 if s["wp"] is None else s["wp"]
    if case["f"]:
        fh = s["f"].float()
        if case["post"] != "none":
            fh, rp = _normed(fh, case["post"])
        x = x + ALPHA * gate * (fh * wp)
        out["x_out"] = x.to(tx)
    if case["pre"] != "none":
        xh, r = _normed(x, case["pre"])
        out["y"] = ((xh * w) * (1.0 + scale) + per_row(s["shift"], 0.0)).to(tb)
    if not case["train"]:
        return out
    dx = s["dx_out"].float()
    if case["pre"] != "none":
        dy = s["dy"].float()
        dx = dx + _normed_back(dy * (1.0 + scale) * w, xh, r, case["pre"])
        dyx = dy * xh
        if s["scale"] is not None:
            out["dscale"] = (over_rows(dyx) * w).float()
            out["dshift"] = over_rows(dy).float()
        if s["w"] is not None:
            out["dweight"] = (dyx * (1.0 + scale)).double().sum(0).float()
    out["dx"] = dx.to(tx)
    if case["f"]:
        dz = ALPHA * gate * dx
        if s["gate"] is not None:
            out["dgate"] = (ALPHA * over_rows(dx * fh) * wp).float()
        if s["wp"] is not None:
            out["dpost_weight"] = (dz * fh).double().sum(0).float()
        e = dz * wp
        out["df"] = (e if case["post"] == "none" else _normed_back(e, fh, rp, case["post"])).to(tb)
    return out


def _act(a, name: str):
    """The activation and its derivative."""
    if name == "silu":
        p = torch.sigmoid(a)
        return a * p, p * (1.0 + a * (1.0 - p))
    c = math.sqrt(2.0 / math.pi)
    t = torch.tanh(c * (a + 0.044715 * a * a * a))
    return 0.5 * a * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * a * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * a * a)


def _ffn_plain(s: Dict) -> Dict:
    case, bf16 = s["case"], torch.bfloat16
    x, wg, wu, wd = (s[k].float() for k in ("x", "wg", "wu", "wd"))
    a, b = x @ wg.T, x @ wu.T
    act, slope = _act(a, case["act"])
    h = act * b
    out = {"y": (h @ wd.T).to(bf16)}
    if not case["train"]:
        return out
    dy = s["dy"].float()
    dh = dy @ wd
    da, db = dh * b * slope, dh * act
    out.update(dx=(da @ wg + db @ wu).to(bf16), dw_gate=(da.T @ x).to(bf16), dw_up=(db.T @ x).to(bf16), dw_down=(dy.T @ h).to(bf16))
    return out


def _clip_plain(s: Dict) -> Dict:
    total = torch.stack([g.double().square().sum() for g in s["grads"]]).sum()
    norm = total.sqrt()
    c = torch.clamp(s["max_norm"] / (norm + CLIP_EPS), max=1.0).float()
    for g, o in zip(s["grads"], s["out"]):
        o.copy_(g.float() * c)
    return {"norm": norm.float(), "grads": list(s["flat"].values())}


def run(state: Dict):
    case = state["case"]
    if not own:
        return {"norm": _norm_plain, "ffn": _ffn_plain, "clip": _clip_plain}[case["op"]](state)
    op = state["op"]
    if case["op"] == "norm":
        x_out, y = op.forward(state["x"], state["f"], gate=state["gate"], scale=state["scale"], shift=state["shift"])
        out = {}
        if case["f"]:
            out["x_out"] = x_out
        if case["pre"] != "none":
            out["y"] = y
        if not case["train"]:
            return out
        out["dx"], df = op.backward(state["x"], state["f"], state["dx_out"], state["dy"], gate=state["gate"], scale=state["scale"])
        if state["scale"] is not None:
            out["dscale"], out["dshift"] = op.dscale, op.dshift
        if state["w"] is not None:
            out["dweight"] = op.dweight
        if case["f"]:
            out["df"] = df
            if state["gate"] is not None:
                out["dgate"] = op.dgate
            if state["wp"] is not None:
                out["dpost_weight"] = op.dpost_weight
        return out
    if case["op"] == "ffn":
        y = op.forward(state["x"])
        if not case["train"]:
            return {"y": y}
        dx, dwg, dwu, dwd = op.backward(state["x"], state["dy"])
        return {"y": y, "dx": dx, "dw_gate": dwg, "dw_up": dwu, "dw_down": dwd}
    return {"norm": op.clip(), "grads": list(state["flat"].values())}


def work(case: Dict) -> Dict:
    if case["op"] == "norm":
        rows, width, n = sum(_lens(case)), case["width"], len(_lens(case))
        sx, sb = (2 if case[k] == "bf16" else 4 for k in ("x", "branch"))
        f, pre = case["f"], case["pre"] != "none"
        vectors = n * (f + 2 * pre) if case["modulated"] else 0
        tensors = sx * (1 + f) + sb * (f + pre)
        if case["train"]:       # dx_out, dy in, dx, df out, and no second reading of x and f
            tensors += 2 * sx + sb * (f + pre)
        return {"bytes": rows * width * tensors + 4 * width * vectors * (2 if case["train"] else 1), "flops": rows * width * (40.0 if case["train"] else 14.0)}
    if case["op"] == "ffn":
        T, D, F = case["tokens"], case["width"], case["hidden"]
        if not case["train"]:
            return {"bytes": 2 * (2 * T * D + 3 * D * F), "flops": 6.0 * T * D * F}
        return {"bytes": 2 * (4 * T * D + 6 * D * F), "flops": 18.0 * T * D * F}
    sizes = _sizes(case)
    total = sum(n * (4 if case["type"] == "fp32" or (case["type"] == "mixed" and i % 3) else 2) for i, n in enumerate(sizes))
    return {"bytes": 2 * total, "flops": 3.0 * sum(sizes)}


def _norm_exact(case: Dict, s: Dict) -> Dict:
    """Sequence by sequence in 64 bits, gradients by automatic differentiation."""
    lens, width, train = _lens(case), case["width"], case["train"]
    leaf = {k: s[k].detach().double().requires_grad_(train) for k in ("x", "f", "gate", "scale", "shift", "w", "wp") if s[k] is not None}
    rows = {"x": torch.split(leaf["x"], lens), "f": torch.split(leaf["f"], lens) if "f" in leaf else None}

    def norm(t, kind):
        if kind == "layer":
            return (t - t.sum(1, keepdim=True) / width) / torch.sqrt(torch.var(t, 1, unbiased=False, keepdim=True) + EPS)
        return t / torch.sqrt((t * t).sum(1, keepdim=True) / width + EPS)

    xs, ys = [], []
    for i in range(len(lens)):
        x = rows["x"][i]
        if case["f"]:
            z = rows["f"][i]
            if case["post"] != "none":
                z = norm(z, case["post"])
            if "wp" in leaf:
                z = z * leaf["wp"]
            if "gate" in leaf:
                z = leaf["gate"][i] * z
            x = x + ALPHA * z
        xs.append(x)
        if case["pre"] != "none":
            y = norm(x, case["pre"])
            if "w" in leaf:
                y = y * leaf["w"]
            if "scale" in leaf:
                y = y + y * leaf["scale"][i] + leaf["shift"][i]
            ys.append(y)
    x_out = torch.cat(xs)
    out = {"x_out": x_out} if case["f"] else {}
    if ys:
        out["y"] = torch.cat(ys)
    if not train:
        return out
    loss = (x_out * s["dx_out"].double()).sum()
    if ys:
        loss = loss + (out["y"] * s["dy"].double()).sum()
    names = {"x": "dx", "f": "df", "gate": "dgate", "scale": "dscale", "shift": "dshift", "w": "dweight", "wp": "dpost_weight"}
    grads = torch.autograd.grad(loss, list(leaf.values()))
    out = {k: v.detach() for k, v in out.items()}
    out.update({names[k]: g for k, g in zip(leaf, grads)})
    return out


def _ffn_exact(case: Dict, s: Dict) -> Dict:
    names = ("x", "wg", "wu", "wd")
    x, wg, wu, wd = (s[k].double().requires_grad_(case["train"]) for k in names)
    a = x.matmul(wg.t())
    if case["act"] == "silu":
        act = a / (1.0 + torch.exp(-a))
    else:       # 0.5 (1 + tanh u) = 1 / (1 + exp(-2 u))
        act = a / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (a + 0.044715 * a ** 3)))
    y = (act * x.matmul(wu.t())).matmul(wd.t())
    if not case["train"]:
        return {"y": y}
    g = torch.autograd.grad(y, (x, wg, wu, wd), s["dy"].double())
    return {"y": y.detach(), "dx": g[0], "dw_gate": g[1], "dw_up": g[2], "dw_down": g[3]}


def _clip_exact(case: Dict, s: Dict) -> Dict:
    norm = math.sqrt(math.fsum(float(torch.dot(g.double(), g.double())) for g in s["grads"]))
    c = min(1.0, s["max_norm"] / (norm + CLIP_EPS))
    flat = []
    for buffer in s["flat"]:
        parts = [torch.nn.functional.pad(g.double() * c, (0, -g.numel() % 64)) for g in s["grads"] if g.dtype == buffer]
        flat.append(torch.cat(parts))
    return {"norm": torch.tensor(norm, dtype=torch.float64, device="cuda"), "grads": flat}


def exact(case: Dict, seed: int):
    s = prepare(case, seed)
    return {"norm": _norm_exact, "ffn": _ffn_exact, "clip": _clip_exact}[case["op"]](case, s)
