"""A first call on another stream than the current one, which is busy: what the classes lay down when they are made is there."""
import pytest

from gpu_util import say


def busy():
    """Work of some ten milliseconds on the current stream."""
    import torch
    a = torch.ones((4096, 4096), device="cuda")
    b = torch.empty_like(a)
    torch.cuda.synchronize()
    for _ in range(60):
        torch.mm(a, a, out=b)


@pytest.mark.gpu
def test_boundaries_and_frequencies_that_were_converted_on_the_gpu():
    import torch
    import paper_2508_06001_amd as K
    say("[gpu] first call on another stream: boundaries of another type")
    rows, width = 300, 264
    cu = torch.tensor([0, 100, 100, 300], device="cuda")
    assert cu.dtype is torch.int64
    x, gate, scale = torch.randn((rows, width), device="cuda"), torch.randn((3, width), device="cuda"), torch.randn((3, width), device="cuda")
    f = torch.randn((rows, width), device="cuda")
    q = torch.randn((rows, 2, 64), device="cuda").bfloat16()
    freq = torch.rand((32,), device="cuda")
    turned = [torch.empty_like(q) for _ in range(4)]
    other = torch.cuda.Stream()

    def run(stream):
        norm = K.ResidualNorm(rows, width, cu, K.KNAP_NORM_RMS, x_type=torch.float32, branch_type=torch.float32)
        norm.forward(x, f, gate, scale, stream=stream)
        rope = K.RotaryPositions(64, K.KNAP_ROPE_HALF, freq, cu_seqlens=cu)
        rope.forward(q, q, *(turned[:2] if stream is None else turned[2:]), stream=stream)
        return norm

    want = run(None)
    torch.cuda.synchronize()
    busy()
    got = run(other)
    torch.cuda.synchronize()
    assert torch.equal(got.x_out, want.x_out) and torch.equal(got.y, want.y)
    assert torch.equal(turned[0], turned[2]) and torch.equal(turned[1], turned[3])
