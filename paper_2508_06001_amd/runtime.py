"""Device-memory plumbing around the two attention entry points.

PyTorch is used for allocation and streams only; the arithmetic is in the
library.  `VarlenAttention` keeps the output, gradient and workspace buffers of
one bag so that repeated calls (benchmark steps, training steps) allocate
nothing.
"""
from __future__ import annotations

from typing import Optional, Sequence

import numpy as np
import torch

from . import binding as B


def bf16_bits_to_device(bits: np.ndarray, device="cuda") -> torch.Tensor:
    """uint16 bf16 bit patterns (host) -> bf16 tensor on the device."""
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).to(device).view(torch.bfloat16)


def bf16_device_to_bits(t: torch.Tensor) -> np.ndarray:
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def _settled(values, dtype, device) -> torch.Tensor:
    """`values` as a tensor on the device, in memory when this returns: a call may go to any stream, and a conversion of values that are on a GPU
    runs on the current one."""
    t = torch.as_tensor(values, dtype=dtype).to(device)
    if t.is_cuda and t is not values and not torch.cuda.is_current_stream_capturing():
        torch.cuda.current_stream(t.device).synchronize()
    return t


class RotaryPositions:
    """Rotary positions of one packed bag: the first `rot` columns of every head turned by `frequencies` (rot / 2 of them, see
    knap_rope_frequencies) times `factor`.  `positions`: int32 (T,) or (T, axes) with the pairs of each axis in `axis_pairs`;
    None for the position in the own sequence of `cu_seqlens`."""

    def __init__(self, rot: int, layout: int, frequencies: Sequence[float], factor: float = 1.0, positions=None, axis_pairs=None,
                 cu_seqlens=None, device="cuda"):
        self.rot, self.layout, self.factor = int(rot), int(layout), float(factor)
        self.freq = _settled(frequencies, torch.float64, device)
        self.positions, self.axis_pairs = positions, list(axis_pairs) if axis_pairs else None
        self.cu = None if cu_seqlens is None else _settled(cu_seqlens, torch.int32, device)

    def forward(self, q, k, q_out, k_out, stream=None):
        B.knap_rope_fwd(q, k, self.rot, self.layout, self.freq, self.factor, q_out, k_out, self.positions, self.axis_pairs, self.cu, stream)
        return q_out, k_out

    def backward(self, dq_out, dk_out, dq, dk, stream=None):
        B.knap_rope_bwd(dq_out, dk_out, self.rot, self.layout, self.freq, self.factor, dq, dk, self.positions, self.axis_pairs, self.cu,
                        stream)
        return dq, dk


class LayerNorm:
    """Buffers + calls of the layer norm of (rows, width) tensors; `weight` and `bias` (width,) or None."""

    def __init__(self, rows: int, width: int, weight=None, bias=None, eps: float = 1e-5, x_type=torch.bfloat16, y_type=torch.bfloat16,
                 train: bool = True, device="cuda"):
        self.rows, self.width, self.eps = int(rows), int(width), float(eps)
        self.weight, self.bias = weight, bias
        self.y = torch.empty((self.rows, self.width), dtype=y_type, device=device)
        self.mean = self.rstd = self.dx = self.dweight = self.dbias = self.workspace = None
        if train:
            self.mean = torch.empty((self.rows,), dtype=torch.float32, device=device)
            self.rstd = torch.empty((self.rows,), dtype=torch.float32, device=device)
            self.dx = torch.empty((self.rows, self.width), dtype=x_type, device=device)
            if weight is not None:
                self.dweight = torch.empty((self.width,), dtype=torch.float32, device=device)
            if bias is not None:
                self.dbias = torch.empty((self.width,), dtype=torch.float32, device=device)
            nbytes = B.knap_layer_norm_bwd_workspace_bytes(self.rows, self.width)
            self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)

    def forward(self, x, stream=None):
        B.knap_layer_norm_fwd(x, self.weight, self.bias, self.eps, self.y, self.mean, self.rstd, stream)
        return self.y

    def backward(self, x, dy, stream=None):
        B.knap_layer_norm_bwd(x, self.weight, self.mean, self.rstd, dy, self.dx, self.dweight, self.dbias, self.workspace, None, stream)
        return self.dx, self.dweight, self.dbias


class ResidualNorm:
    """Buffers + calls of the norms around a branch (knap_residual_norm_fwd) over the rows of a packed bag: `post_norm` with `post_weight` behind
    the branch, the residual scale `alpha`, `norm` with `weight` in front of the next branch.  `cu_seqlens` None: one sequence of all rows.
    `branch=False`: a block's first norm, without a residual.  Gradients of the vectors are in `dgate`, `dscale` and `dshift`, those of the
    weights in `dweight` and `dpost_weight`."""

    def __init__(self, rows: int, width: int, cu_seqlens=None, norm: int = B.KNAP_NORM_LAYER, weight=None, post_norm: int = B.KNAP_NORM_NONE,
                 post_weight=None, alpha: float = 1.0, eps: float = 1e-6, x_type=torch.bfloat16, branch_type=torch.bfloat16, branch: bool = True,
                 train: bool = True, device="cuda"):
        self.rows, self.width, self.alpha, self.eps = int(rows), int(width), float(alpha), float(eps)
        self.norm, self.weight, self.post_norm, self.post_weight = norm, weight, post_norm, post_weight
        self.cu = None if cu_seqlens is None else _settled(cu_seqlens, torch.int32, device)
        self.n_seq = 1 if self.cu is None else self.cu.numel() - 1
        self.branch = bool(branch)
        normed = norm != B.KNAP_NORM_NONE

        def new(there, dtype, *shape):
            return torch.empty(shape or (self.rows, self.width), dtype=dtype, device=device) if there else None

        f32 = torch.float32
        self.x_out, self.y = new(branch, x_type), new(normed, branch_type)
        self.stats = new(train, f32, 4, self.rows)
        self.dx, self.df = new(train, x_type), new(train and branch, branch_type)
        vectors = (self.n_seq, self.width)
        self._dgate = new(train and branch, f32, *vectors)
        self._dscale, self._dshift = new(train and normed, f32, *vectors), new(train and normed, f32, *vectors)
        self.dgate = self.dscale = self.dshift = None
        self.dweight, self.dpost_weight = new(train and weight is not None, f32, self.width), new(train and post_weight is not None, f32, self.width)
        self.workspace = None
        if train:
            nbytes = B.knap_residual_norm_bwd_workspace_bytes(self.rows, self.width, self.n_seq)
            self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)

    def forward(self, x, f=None, gate=None, scale=None, shift=None, stream=None):
        """x_out (x itself without a branch) and y (None without a norm)."""
        B.knap_residual_norm_fwd(x, f, self.x_out, self.y, self.norm, self.post_norm, self.weight, self.post_weight, gate, scale, shift, self.cu,
                                 self.alpha, self.eps, self.stats, stream)
        return (self.x_out if self.branch else x), self.y

    def backward(self, x, f, dx_out, dy, gate=None, scale=None, shift=None, stream=None):
        """dx and df (None without a branch); x, f, gate and scale as the forward had them.  dgate is formed where a gate is given, dscale where
        a scale is, dshift where a scale or a shift is."""
        self.dgate = self._dgate if gate is not None else None
        self.dscale = self._dscale if scale is not None else None
        self.dshift = self._dshift if scale is not None or shift is not None else None
        B.knap_residual_norm_bwd(x, f, self.stats, dx_out, dy, self.dx, self.df, self.norm, self.post_norm, self.weight, self.post_weight, gate, scale,
                                 self.cu, self.alpha, self.dgate, self.dscale, self.dshift, self.dweight, self.dpost_weight, self.workspace, None,
                                 stream)
        return self.dx, self.df


class GatedFeedForward:
    """Buffers + calls of the gated feed-forward block of (tokens, width) rows: y = (act(x w_gate^T) (x w_up^T)) w_down^T."""

    def __init__(self, tokens: int, width: int, hidden: int, w_gate, w_up, w_down, act: int = B.KNAP_SILU, train: bool = True, device="cuda"):
        self.tokens, self.width, self.hidden, self.act = int(tokens), int(width), int(hidden), act
        self.w_gate, self.w_up, self.w_down = w_gate, w_up, w_down

        def new(*shape):
            return torch.empty(shape, dtype=torch.bfloat16, device=device)

        self.y, self.h = new(self.tokens, self.width), new(self.tokens, self.hidden)
        self.gate = self.up = self.dx = self.dw_gate = self.dw_up = self.dw_down = None
        nbytes = B.knap_gated_ffn_fwd_workspace_bytes(self.tokens, self.width, self.hidden)
        if train:
            self.gate, self.up, self.dx = new(self.tokens, self.hidden), new(self.tokens, self.hidden), new(self.tokens, self.width)
            self.dw_gate, self.dw_up, self.dw_down = new(self.hidden, self.width), new(self.hidden, self.width), new(self.width, self.hidden)
            nbytes = max(nbytes, B.knap_gated_ffn_bwd_workspace_bytes(self.tokens, self.width, self.hidden))
        self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)

    def forward(self, x, stream=None):
        B.knap_gated_ffn_fwd(x, self.w_gate, self.w_up, self.w_down, self.act, self.gate, self.up, self.h, self.y, self.workspace, None, stream)
        return self.y

    def backward(self, x, dy, stream=None):
        B.knap_gated_ffn_bwd(x, self.w_gate, self.w_up, self.w_down, self.act, self.gate, self.up, self.h, dy, self.dx, self.dw_gate, self.dw_up,
                             self.dw_down, self.workspace, None, stream)
        return self.dx, self.dw_gate, self.dw_up, self.dw_down


class GradientClip:
    """Buffers + calls of the global norm of a fixed list of gradients and clipping by it, in place or into `out`.  Ranks that hold parts of the
    gradients call sum_squares, add up `sum_sq` (an all-reduce of one float64) and call scale; clip does both on one GPU.
    The plan points to the gradients' memory as it was laid down, which this object keeps.  A program whose gradients are other tensors from step to
    step (set to None in between) asks stands_for, or copies them to ones that stay."""

    def __init__(self, grads, max_norm: float, eps: float = 1e-6, out=None):
        self.grads = list(grads)
        self.out = self.grads if out is None else list(out)
        self.plan = B.knap_grad_plan(self.grads, self.out)
        # tensors of their own on the same memory: a caller's tensor may be given other memory, and what it had would be freed under the plan
        self._held = [t.detach() for t in self.grads]
        self._held_out = [] if out is None else [t.detach() for t in self.out]
        self.max_norm, self.eps = float(max_norm), float(eps)
        device = self.plan.device
        # not filled here: a fill would still be under way when the first call runs on another stream
        self.sum_sq = torch.empty((), dtype=torch.float64, device=device)
        self.norm = torch.empty((), dtype=torch.float32, device=device)
        self.workspace = torch.empty(B.KNAP_GRAD_WORKSPACE_BYTES, dtype=torch.uint8, device=device)

    def stands_for(self, grads) -> bool:
        """Whether these are the gradients that the plan was laid down for, where they were then."""
        grads = list(grads)
        return len(grads) == len(self._held) and all(
            g is not None and g.data_ptr() == h.data_ptr() and g.numel() == h.numel() and g.dtype is h.dtype for g, h in zip(grads, self._held))

    def sum_squares(self, stream=None):
        B.knap_grad_sum_squares(self.plan, self.sum_sq, self.workspace, B.KNAP_GRAD_WORKSPACE_BYTES, stream)
        return self.sum_sq

    def scale(self, stream=None):
        B.knap_grad_clip(self.plan, self.sum_sq, self.max_norm, self.eps, self.norm, stream)
        return self.norm

    def clip(self, stream=None):
        """The norm as it was before."""
        self.sum_squares(stream)
        return self.scale(stream)


class VarlenAttention:
    """Buffers + calls for one packed bag: T tokens, H heads, head dim d; `causal` selects the
    causal pair of entry points; `rope`, a RotaryPositions, turns q and k in front of the attention
    and their gradients back behind it."""

    def __init__(self, cu_seqlens: Sequence[int], H: int, d: int, scale: float, device="cuda",
                 causal: bool = False, rope: Optional[RotaryPositions] = None):
        self.causal = bool(causal)
        self.rope = rope
        cu = np.asarray(cu_seqlens, dtype=np.int32)
        self.n_seq = int(cu.shape[0] - 1)
        self.T = int(cu[-1]) if cu.shape[0] else 0
        self.H, self.d, self.scale = int(H), int(d), float(scale)
        self.device = torch.device(device)
        self.cu = torch.from_numpy(cu).to(self.device)
        shape = (self.T, self.H, self.d)
        self.out = torch.empty(shape, dtype=torch.bfloat16, device=self.device)
        self.lse = torch.empty((self.H, self.T), dtype=torch.float32, device=self.device)
        self.dq = self.dk = self.dv = None
        self.workspace = None
        if rope is not None:
            self.q_turned = torch.empty(shape, dtype=torch.bfloat16, device=self.device)
            self.k_turned = torch.empty(shape, dtype=torch.bfloat16, device=self.device)

    def forward(self, q, k, v, stream=None):
        if self.rope is not None:
            q, k = self.rope.forward(q, k, self.q_turned, self.k_turned, stream)
        fwd = B.knap_varlen_attn_causal_fwd if self.causal else B.knap_varlen_attn_fwd
        fwd(q, k, v, self.cu, self.n_seq, self.H, self.d, self.scale, self.out, self.lse, stream)
        return self.out, self.lse

    def _ensure_bwd_buffers(self):
        if self.dq is None:
            shape = (self.T, self.H, self.d)
            self.dq = torch.empty(shape, dtype=torch.bfloat16, device=self.device)
            self.dk = torch.empty(shape, dtype=torch.bfloat16, device=self.device)
            self.dv = torch.empty(shape, dtype=torch.bfloat16, device=self.device)
            nbytes = B.knap_varlen_attn_bwd_workspace_bytes(self.T, self.n_seq, self.H, self.d)
            self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.device)

    def backward(self, q, k, v, dout, stream=None):
        self._ensure_bwd_buffers()
        if self.rope is not None:        # as the forward left them
            q, k = self.q_turned, self.k_turned
        bwd = B.knap_varlen_attn_causal_bwd if self.causal else B.knap_varlen_attn_bwd
        bwd(q, k, v, self.cu, self.n_seq, self.H, self.d, self.scale, self.out, self.lse, dout,
            self.dq, self.dk, self.dv, self.T, self.workspace, None, stream)
        if self.rope is not None:
            self.rope.backward(self.dq, self.dk, self.dq, self.dk, stream)
        return self.dq, self.dk, self.dv


class VarlenDiffAttention:
    """Buffers + calls of differential attention over one packed bag: `lam` is the fp32 (H,) weight of the second map; `train=False`
    keeps nothing for a backward.  `rope` turns the q and k of each map in front, as heads of d / 2 columns (rot <= d / 2).  `norm`, a
    LayerNorm of T * H rows of d, is applied to every head's output row behind the difference."""

    def __init__(self, cu_seqlens: Sequence[int], H: int, d: int, scale: float, lam, device="cuda", causal: bool = False, train: bool = True,
                 rope: Optional[RotaryPositions] = None, norm: Optional[LayerNorm] = None):
        self.causal, self.rope, self.norm = bool(causal), rope, norm
        cu = np.asarray(cu_seqlens, dtype=np.int32)
        self.n_seq = int(cu.shape[0] - 1)
        self.T = int(cu[-1]) if cu.shape[0] else 0
        self.H, self.d, self.scale, self.lam = int(H), int(d), float(scale), lam
        self.device = torch.device(device)
        self.cu = torch.from_numpy(cu).to(self.device)
        shape = (self.T, self.H, self.d)

        def new():
            return torch.empty(shape, dtype=torch.bfloat16, device=self.device)

        self.out = new()
        self.lse = torch.empty((2, self.H, self.T), dtype=torch.float32, device=self.device)
        self.out2 = self.dq = self.dk = self.dv = self.dlam = self.workspace = None
        if train:
            self.out2, self.dq, self.dk, self.dv = new(), new(), new(), new()
            # not filled here, but for no sequences, where a backward writes nothing: a fill that is still under way when a backward runs on
            # another stream would put zeros over its result
            self.dlam = (torch.empty if self.n_seq else torch.zeros)((self.H,), dtype=torch.float32, device=self.device)
            nbytes = B.knap_varlen_diff_attn_bwd_workspace_bytes(self.T, self.n_seq, self.H, self.d)
            self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.device)
        if rope is not None:
            self.q_turned, self.k_turned = new(), new()

    def _maps(self, *tensors):
        return [t.view(self.T, 2 * self.H, self.d // 2) for t in tensors]

    def forward(self, q, k, v, stream=None):
        if self.rope is not None:
            self.rope.forward(*self._maps(q, k, self.q_turned, self.k_turned), stream)
            q, k = self.q_turned, self.k_turned
        fwd = B.knap_varlen_diff_attn_causal_fwd if self.causal else B.knap_varlen_diff_attn_fwd
        fwd(q, k, v, self.cu, self.n_seq, self.H, self.d, self.scale, self.lam, self.out, self.out2, self.lse, stream)
        if self.norm is None:
            return self.out, self.lse
        return self.norm.forward(self.out.view(self.T * self.H, self.d), stream).view(self.T, self.H, self.d), self.lse

    def backward(self, q, k, v, dout, stream=None):
        """dq, dk, dv, dlambda; the norm's own gradients are in `norm.dweight` and `norm.dbias`."""
        if self.norm is not None:
            rows = self.T * self.H
            dout = self.norm.backward(self.out.view(rows, self.d), dout.view(rows, self.d), stream)[0].view(self.T, self.H, self.d)
        if self.rope is not None:        # as the forward left them
            q, k = self.q_turned, self.k_turned
        bwd = B.knap_varlen_diff_attn_causal_bwd if self.causal else B.knap_varlen_diff_attn_bwd
        bwd(q, k, v, self.cu, self.n_seq, self.H, self.d, self.scale, self.lam, self.out, self.out2, self.lse, dout, self.dq, self.dk, self.dv,
            self.dlam, self.T, self.workspace, None, stream)
        if self.rope is not None:
            grads = self._maps(self.dq, self.dk)
            self.rope.backward(*grads, *grads, stream)
        return self.dq, self.dk, self.dv, self.dlam
