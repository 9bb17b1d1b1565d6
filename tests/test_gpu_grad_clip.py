"""Global gradient norm and clipping against sums in 64 bits: lists of every make-up, sizes around a chunk and a 16-byte unit, offsets, types,
in place and not, large values and values that are not finite; and refusals.

Bars.  The sum of squares runs in 64 bits: up to 2^40 squares, each off by 2^-53, added up in a tree of chains far shorter than 2^20, so that
2^-30 of the sum is far above what may be lost, and the norm is rounded once to 32 bits (2^-24).  The factor is rounded to 32 bits, the
product again, and then to its type: (2^-22 + half a step) of the value, and below the least normal number the steps there."""
import math

import numpy as np
import pytest

from gpu_util import say

HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
LEAST = 2.0 ** -126 * 2.0 ** -7       # a step of bf16 below its least normal number, which 32 bits have as well


def tensors(sizes, types, shift=0, seed=0, scale=None):
    """Gradients that start `shift` elements behind 16 bytes."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, (n, t) in enumerate(zip(sizes, types)):
        v = torch.randn((n + shift,), generator=g, device="cuda") * (10.0 ** (i % 5 - 3) if scale is None else scale)
        out.append(v.to({"bf16": torch.bfloat16, "fp32": torch.float32}[t])[shift:])
    return out


def name_of(t):
    return "bf16" if t.element_size() == 2 else "fp32"


def exact_norm(grads):
    return math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in grads))


def check(before, out, norm, max_norm, eps):
    want = exact_norm(before)
    if want < 3.4e38:
        assert abs(norm - want) <= (2.0 ** -24 + 2.0 ** -30) * want + 2.0 ** -149, (norm, want)
    else:       # the norm as 32 bits have it; the factor is formed from the sum in 64
        assert norm == math.inf
    c = min(1.0, max_norm / (want + eps))
    for i, (g, o) in enumerate(zip(before, out)):
        ref = g.double() * c
        assert bool(((o.double() - ref).abs() <= (2.0 ** -22 + HALF[name_of(g)]) * ref.abs() + LEAST).all()), i


def clip(grads, max_norm, eps=1e-6, out=None):
    import torch
    import paper_2508_06001_amd as K
    c = K.GradientClip(grads, max_norm, eps, out)
    c.workspace.fill_(255)
    norm = c.clip()
    torch.cuda.synchronize()
    assert c.norm is norm
    return float(norm)


SIZES = {"one": [1], "few": [3, 8191, 8192, 8193, 1, 0, 16384, 100000], "none": [], "empty": [0, 0], "large": [5_000_011, 7],
         "many": [1 + 37 * i for i in range(113)], "more": [1 + (i * i) % 9001 for i in range(400)], "odd": [7, 9, 15, 17, 4095, 4097]}


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "fp32", "mixed"])
@pytest.mark.parametrize("name", list(SIZES))
def test_lists(name, kind):
    import torch
    sizes = SIZES[name]
    types = [kind if kind != "mixed" else ("fp32", "bf16", "bf16")[i % 3] for i in range(len(sizes))]
    for shift in (0, 1, 3):
        say(f"[gpu] clip {name} {kind} shift={shift}")
        grads = tensors(sizes, types, shift)
        want = exact_norm(grads)
        for factor in (0.1, 3.0):
            before = [g.clone() for g in grads]
            apart = [torch.full_like(g, float("nan")) for g in grads]
            norm = clip(before, factor * want + 1e-3, out=apart)
            check(grads, apart, norm, factor * want + 1e-3, 1e-6)
            assert all(torch.equal(a, b) for a, b in zip(grads, before))
            assert clip(before, factor * want + 1e-3) == norm
            assert all(torch.equal(a, b) for a, b in zip(before, apart))


@pytest.mark.gpu
def test_no_neighbour_is_touched_and_the_same_call_has_the_same_bits():
    import torch
    import paper_2508_06001_amd as K
    for dtype in (torch.bfloat16, torch.float32):
        flat = torch.randn((100_000,), device="cuda").to(dtype)
        keep = flat.clone()
        parts = [flat[1:8194], flat[8200:8201], flat[9000:50_001]]
        c = K.GradientClip(parts, 1.0)
        first = float(c.clip())
        touched = torch.zeros((100_000,), dtype=torch.bool, device="cuda")
        for a, b in ((1, 8194), (8200, 8201), (9000, 50_001)):
            touched[a:b] = True
        assert torch.equal(flat[~touched], keep[~touched]) and bool((flat[touched].abs() <= keep[touched].abs()).all())
        flat.copy_(keep)
        c.workspace.fill_(127)
        assert float(c.clip()) == first


@pytest.mark.gpu
def test_large_small_and_not_finite():
    import torch
    import paper_2508_06001_amd as K
    for scale in (1e30, 1e-30, 3e37):       # squares past the range of 32 bits on both sides
        grads = tensors([5000, 77], ["fp32", "bf16"], scale=scale)
        before = [g.clone() for g in grads]
        check(before, grads, clip(grads, scale, eps=0.0), scale, 0.0)
    zero = [torch.zeros((100,), device="cuda")]
    assert clip(zero, 1.0) == 0.0 and not bool(zero[0].any())
    nan = tensors([100, 50], ["fp32", "bf16"])
    nan[1][3] = float("nan")
    assert math.isnan(clip(nan, 1.0)) and all(bool(torch.isnan(g).all()) for g in nan)
    inf = tensors([100, 50], ["fp32", "bf16"])
    inf[0][99] = float("-inf")
    assert clip(inf, 1.0) == math.inf
    assert bool(torch.isnan(inf[0][99])) and not bool(inf[0][:99].any()) and not bool(inf[1].any())
    free = tensors([100, 50], ["fp32", "bf16"])
    keep = [g.clone() for g in free]
    check(keep, free, clip(free, math.inf), math.inf, 1e-6)
    assert all(torch.equal(a, b) for a, b in zip(free, keep))
    c = K.GradientClip(keep, 1e-3)
    c.sum_squares()
    c.sum_sq.mul_(4.0)                      # as an all-reduce over four ranks of the same gradients would leave it
    half = float(c.scale())
    assert half == pytest.approx(2 * exact_norm(free), rel=1e-6)
    check([g * 2 for g in free], [g * 2 for g in keep], half, 1e-3, 1e-6)


@pytest.mark.gpu
def test_a_tensor_past_two_to_the_32_bytes():
    import torch
    n = (1 << 31) + 12345
    say("[gpu] clip of 2^31 elements")
    big = torch.zeros((n,), dtype=torch.bfloat16, device="cuda")
    big[-5:] = 3.0
    big[0] = 2.0
    norm = clip([big], 0.5, eps=0.0)
    assert norm == 7.0 and bool((big[-5:] == torch.tensor(3.0 / 14, dtype=torch.bfloat16)).all()) and not bool(big[1:-5].any())


@pytest.mark.gpu
def test_captured_calls_follow_the_gradients():
    import torch
    import paper_2508_06001_amd as K
    sizes, types = [100_003, 5, 64], ["bf16", "fp32", "bf16"]
    grads, eager = tensors(sizes, types), tensors(sizes, types)
    a, b = K.GradientClip(grads, 1.0), K.GradientClip(eager, 1.0)
    b.clip()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        a.clip()
    for turn in range(4):
        for g, e in zip(grads, eager):
            g.normal_().mul_(10.0 ** (turn - 2))
            e.copy_(g)
        graph.replay()
        b.clip()
        torch.cuda.synchronize()
        assert float(a.norm) == float(b.norm) and all(torch.equal(g, e) for g, e in zip(grads, eager)), turn


@pytest.mark.gpu
def test_at_once_on_another_stream_than_the_current_one():
    import torch
    import paper_2508_06001_amd as K
    other = torch.cuda.Stream()
    grads = tensors([50_001, 3, 8192], ["fp32", "bf16", "bf16"])
    before = [g.clone() for g in grads]
    want = clip([g.clone() for g in grads], 1.0)
    for turn in range(20):
        for g, b in zip(grads, before):
            g.copy_(b)
        torch.cuda.synchronize()
        c = K.GradientClip(grads, 1.0)
        c.clip(stream=other)
        torch.cuda.synchronize()
        assert float(c.norm) == want, turn
        check(before, grads, want, 1.0, 1e-6)


def arrays(at, numel, types):
    import ctypes as C
    n = max(1, len(at))
    return (C.c_void_p * n)(*at), (C.c_int64 * n)(*numel), (C.c_int * n)(*types)


def test_bad_arguments_are_refused_without_touching_a_gpu():
    import ctypes as C
    import paper_2508_06001_amd as K
    bad = K.KNAP_ERR_INVALID_ARG
    room = (C.c_uint64 * 3000)()

    def plan(at=(4096, 8192), out=(16384, 32768), numel=(8, 8), types=(0, 1), n=2, to=room, size=None):
        a, m, t = arrays(at, numel, types)
        return K.lib.knap_grad_plan(a, arrays(out, numel, types)[0], m, t, n, C.cast(to, C.c_void_p) if to is not None else 0,
                                    C.sizeof(room) if size is None else size)

    assert plan() == K.KNAP_OK and plan(at=(4096, 0), out=(0, 0), numel=(0, 0)) == K.KNAP_OK and plan(n=0, to=None) == K.KNAP_OK
    assert plan(at=(4096, 8192), out=(4096, 8192)) == K.KNAP_OK and plan(at=(4096, 4096), types=(1, 1)) == K.KNAP_OK      # read twice: as it says
    for wrong in (dict(n=-1), dict(at=(0, 8192)), dict(at=(4097, 8192)), dict(at=(4096, 8194)), dict(out=(0, 32768)), dict(out=(16385, 32768)),
                  dict(numel=(-1, 8)), dict(numel=(1 << 40, 8)), dict(types=(2, 0)), dict(types=(0, -1)), dict(to=None),
                  dict(at=(4096, 4096), out=(4096, 4096), types=(1, 1)),            # a tensor twice
                  dict(out=(16384, 16392)), dict(out=(16392, 16384)),               # parts of out that overlap
                  dict(out=(4096, 8176)), dict(out=(8192, 4096)), dict(out=(4104, 32768)), dict(out=(16384, 4096))):      # and that overlap a gradient
        assert plan(**wrong) == bad, wrong
    assert plan(size=47) == K.KNAP_ERR_CAPACITY
    many = 600           # more than the space on the stack holds: in order, in reverse order, one of them twice
    up = [4096 + 64 * i for i in range(many)]
    again = up[:-1] + [up[3]]
    assert plan(at=again, out=again, numel=[8] * many, types=[1] * many, n=many) == bad
    shifted = [a + 16 for a in up[::-1]]
    assert plan(at=up[::-1], out=shifted, numel=[8] * many, types=[1] * many, n=many) == bad
    assert plan(at=up[::-1], out=up[::-1], numel=[8] * many, types=[1] * many, n=many) == K.KNAP_OK
    assert K.lib.knap_grad_plan_bytes(0, 5) == 0
    squares = lambda p=256, size=48, s=256, ws=256, n=8192: K.lib.knap_grad_sum_squares(p, size, s, ws, n, 0)  # noqa: E731
    scale = lambda p=256, size=48, s=256, top=1.0, eps=0.0, norm=256: K.lib.knap_grad_clip(p, size, s, top, eps, norm, 0)  # noqa: E731
    for wrong in (dict(p=0), dict(p=260), dict(size=47), dict(s=0), dict(s=260), dict(ws=0), dict(ws=128)):
        assert squares(**wrong) == bad, wrong
    assert squares(n=K.KNAP_GRAD_WORKSPACE_BYTES - 1) == K.KNAP_ERR_WORKSPACE_TOO_SMALL
    nan, inf = float("nan"), float("inf")
    for wrong in (dict(p=0), dict(p=4), dict(size=100), dict(s=0), dict(s=4), dict(top=0.0), dict(top=-1.0), dict(top=nan), dict(eps=-1.0), dict(eps=nan),
                  dict(eps=inf), dict(norm=2)):
        assert scale(**wrong) == bad, wrong
    assert scale(p=0, size=0, norm=0) == K.KNAP_OK


def test_a_plan_covers_every_element_once():
    """Walks through the records as the kernels do."""
    import ctypes as C
    import paper_2508_06001_amd as K
    numel = [1, 0, 8191, 8192, 8193, 5, 3 * 8192 + 17]
    types = [0, 1, 1, 0, 1, 0, 1]
    at = [1 << 20, 0, 2 << 20, 3 << 20, 4 << 20, 5 << 20, 6 << 20]
    to = [a + (64 << 20) for a in at]
    a, m, t = arrays(at, numel, types)
    size = K.lib.knap_grad_plan_bytes(m, len(numel))
    buf = (C.c_uint8 * size)()
    assert K.lib.knap_grad_plan(a, arrays(to, numel, types)[0], m, t, len(numel), C.cast(buf, C.c_void_p), size) == K.KNAP_OK
    records = np.frombuffer(bytes(buf), dtype=[("from", "<u8"), ("to", "<u8"), ("count", "<i4"), ("bf16", "<i4")])
    i = 0
    for n, ty, g, o in zip(numel, types, at, to):
        done, width = 0, 2 if ty == 0 else 4
        while done < n:
            r = records[i]
            i += 1
            assert r["from"] == g + done * width and r["to"] == o + done * width and r["bf16"] == (ty == 0) and 0 < r["count"] <= K.KNAP_GRAD_CHUNK
            done += int(r["count"])
        assert done == n
    assert i == len(records)


@pytest.mark.gpu
def test_the_binding_refuses_what_the_library_cannot_see():
    import torch
    import paper_2508_06001_amd as K
    g = torch.zeros((8, 8), device="cuda")
    s, ws = torch.zeros((), dtype=torch.float64, device="cuda"), torch.empty((1 << 16,), dtype=torch.uint8, device="cuda")
    plan = K.knap_grad_plan([g])
    K.knap_grad_sum_squares(plan, s, ws)
    K.knap_grad_clip(plan, s, 1.0)
    for grads, out in (([g.half()], None), ([g.t()[:, :4]], None), ([g], []), ([g], [g.bfloat16()]), ([g], [g[:4]]), ([g.cpu(), g], None), ([g, g], None),
                       ([g, g[:4]], None)):
        with pytest.raises(K.KnapError):
            K.knap_grad_plan(grads, out)
    for args in ((plan, s.float(), ws), (plan, s, None), (plan, s, ws[:64]), (plan, s.cpu(), ws), (plan.cpu(), s, ws), (plan.view(torch.int32), s, ws),
                 (plan[:23], s, ws), (plan, s.new_zeros(2), ws)):
        with pytest.raises(K.KnapError):
            K.knap_grad_sum_squares(*args)
    for args, kw in (((plan, s, 0.0), {}), ((plan, s, 1.0), dict(norm=s)), ((plan.cpu(), s, 1.0), {}), ((plan, s.float(), 1.0), {})):
        with pytest.raises(K.KnapError):
            K.knap_grad_clip(*args, **kw)
