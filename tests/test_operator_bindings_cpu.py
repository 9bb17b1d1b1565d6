"""What the binding lets through to the operators around attention, without a GPU: CPU tensors, the library's function replaced by one that
counts its calls."""
import pytest
import torch

import paper_2508_06001_amd as K
from paper_2508_06001_amd import binding as B


@pytest.fixture
def calls(monkeypatch):
    """Names of the library's functions that were reached."""
    reached = []
    monkeypatch.setattr(B, "_here", lambda *a: None)
    for name in B.EXPORTS:
        if name.startswith(("knap_varlen_diff_attn", "knap_rope_fwd", "knap_rope_bwd")) and not name.endswith("workspace_bytes"):
            monkeypatch.setattr(B.lib, name, lambda *a, name=name: reached.append(name) or 0)
    return reached


T, H, d = 10, 2, 64


def diff_args(rows=T, backward=False):
    new = lambda: torch.zeros((rows, H, d), dtype=torch.bfloat16)  # noqa: E731
    args = dict(q=new(), k=new(), v=new(), cu_seqlens=torch.tensor([0, 4, T], dtype=torch.int32), n_seq=2, H=H, d=d, scale=0.1, lam=torch.zeros((H,)),
                out=new(), out2=new(), lse=torch.zeros((2, H, T)), stream=0)
    if backward:
        args.update(dout=new(), dq=new(), dk=new(), dv=new(), dlam=torch.zeros((H,)), total_tokens=T, workspace=torch.zeros((1 << 16,), dtype=torch.uint8))
    return args


DIFF = [(K.knap_varlen_diff_attn_fwd, False), (K.knap_varlen_diff_attn_causal_fwd, False), (K.knap_varlen_diff_attn_bwd, True),
        (K.knap_varlen_diff_attn_causal_bwd, True)]


@pytest.mark.parametrize("fn,backward", DIFF)
def test_log_sums_of_differential_attention_have_room(calls, fn, backward):
    """2 H T of them are written, T being known on the device alone: at least as many as q has rows, or a (2, H, T) tensor of a padded bag.
    The (H, T) tensor of plain attention holds half of them."""
    for rows, lse in ((T, torch.zeros((2, H, T))), (T + 7, torch.zeros((2, H, T))), (T + 7, torch.zeros((2 * H * (T + 7),))), (T, torch.zeros((3 * H * T,)))):
        fn(**{**diff_args(rows, backward), "lse": lse})
    assert len(calls) == 4
    for rows, lse in ((T, torch.zeros((H, T))), (T, torch.zeros((1, H, T))), (T, torch.zeros((0,))), (T, torch.zeros((2 * H * T - 1,))),
                      (T, torch.zeros((2, H, 2 * T))[..., :T]), (T, torch.zeros((2, H, T), dtype=torch.float64)), (T + 7, torch.zeros((H, T + 7)))):
        with pytest.raises(K.KnapError):
            fn(**{**diff_args(rows, backward), "lse": lse})
    assert len(calls) == 4


@pytest.mark.parametrize("fn,backward", DIFF)
def test_rows_of_differential_attention_are_of_h_heads_of_d(calls, fn, backward):
    """The kernels go by H and d: tensors of other heads, of another d, of another order or with fewer rows are refused."""
    fn(**diff_args(backward=backward))
    flat = diff_args(backward=backward)
    fn(**{n: t.view(T, H * d) if torch.is_tensor(t) and t.dim() == 3 and t.dtype is torch.bfloat16 else t for n, t in flat.items()})
    assert len(calls) == 2
    wrong = [dict(H=3), dict(H=1), dict(d=128), dict(H=1, d=128), dict(H=4, d=32), dict(H=2 * H, lam=torch.zeros((2 * H,))), dict(q=None)]
    names = ["k", "v", "out", "out2"] + (["dout", "dq", "dk", "dv"] if backward else [])
    for n in names:
        wrong += [{n: torch.zeros((T - 1, H, d), dtype=torch.bfloat16)}, {n: torch.zeros((H, T, d), dtype=torch.bfloat16)},
                  {n: torch.zeros((T, d, H), dtype=torch.bfloat16)}]
    for w in wrong:
        with pytest.raises(K.KnapError):
            fn(**{**diff_args(backward=backward), **w})
    assert len(calls) == 2


@pytest.mark.parametrize("fn", [K.knap_rope_fwd, K.knap_rope_bwd])
def test_rotary_positions_have_an_axis(calls, fn):
    """A tensor of positions without an axis has no address, which the library takes for none given: nothing would be turned."""
    x = torch.zeros((T, H, d), dtype=torch.bfloat16)
    call = lambda pos, **kw: fn(x, None, d, K.KNAP_ROPE_HALF, torch.ones((d // 2,), dtype=torch.float64), 1.0, torch.empty_like(x), None,  # noqa: E731
                                positions=pos, stream=0, **kw)
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    call(ints(T))
    call(ints(T, 1))
    call(ints(T, 2), axis_pairs=[16, 16])
    assert len(calls) == 3
    for wrong in (ints(T, 0), ints(), ints(T, 2, 0)):
        with pytest.raises(K.KnapError):
            call(wrong)
    assert len(calls) == 3
