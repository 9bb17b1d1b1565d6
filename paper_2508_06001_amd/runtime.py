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


class RotaryPositions:
    """Rotary positions of one packed bag: the first `rot` columns of every head turned by `frequencies` (rot / 2 of them, see
    knap_rope_frequencies) times `factor`.  `positions`: int32 (T,) or (T, axes) with the pairs of each axis in `axis_pairs`;
    None for the position in the own sequence of `cu_seqlens`."""

    def __init__(self, rot: int, layout: int, frequencies: Sequence[float], factor: float = 1.0, positions=None, axis_pairs=None,
                 cu_seqlens=None, device="cuda"):
        self.rot, self.layout, self.factor = int(rot), int(layout), float(factor)
        self.freq = torch.as_tensor(frequencies, dtype=torch.float64).to(device)
        self.positions, self.axis_pairs = positions, list(axis_pairs) if axis_pairs else None
        self.cu = None if cu_seqlens is None else torch.as_tensor(cu_seqlens, dtype=torch.int32).to(device)

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
            self.dlam = torch.zeros((self.H,), dtype=torch.float32, device=self.device)
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
