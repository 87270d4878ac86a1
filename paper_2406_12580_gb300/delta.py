"""The gated delta rule as a torch operator, and the recurrent layer around it.

    S~ = exp(g_t) S_{t-1},  u_t = beta_t (v_t - S~^T k_t),  S_t = S~ + k_t u_t^T,  o_t = scale S_t^T q_t

``gated_delta_rule`` runs whole sequences with gradients for every input,
``blr_gdr_steps`` single steps on kept states; both on the library's kernels.
``GatedDeltaLayer`` is the gated recurrent layer with this recurrence in the
BD-LRU's place: decay and write strength are computed from the same inputs,
and a step form serves a trained layer with O(1) work per new behavior.
"""
from __future__ import annotations

import math
from typing import Optional

import torch
from torch import nn

from . import (BLR_F32, BLR_GDR_STATE, BLR_GDR_TRAIN, GDRDesc, _dtype_code, blr_gdr_bwd, blr_gdr_fwd,
               blr_gdr_steps, blr_gdr_workspace_bytes)


def _rows(t: torch.Tensor) -> torch.Tensor:
    """t (B, L, H, D) itself when its steps lie at one distance (a slice of wider rows), else a copy."""
    B, L, H, D = t.shape
    s = t.stride()
    ld = s[1] if L > 1 else H * D
    fits = (s[3] == 1 and (H == 1 or s[2] == D) and ld >= H * D and ld % 8 == 0
            and (B == 1 or s[0] == L * ld) and t.data_ptr() % 16 == 0)
    return t if fits else t.contiguous()


def _prepare(q, k, v, g, beta, scale, s0, lengths):
    if q.dim() != 4 or k.shape != q.shape or v.dim() != 4 or v.shape[:2] != q.shape[:2]:
        raise ValueError("q and k (B, L, Hk, Dk) and v (B, L, Hv, Dv) are wanted")
    if g.shape != v.shape[:3] or beta.shape != v.shape[:3]:
        raise ValueError("g and beta (B, L, Hv) are wanted")
    if any(t.dtype != v.dtype for t in (q, k, g, beta)):
        raise TypeError("q, k, v, g and beta must have one dtype")
    B, L, Hk, Dk = q.shape
    Hv, Dv = v.shape[2:]
    if s0 is not None and (s0.shape != (B, Hv, Dk, Dv) or s0.dtype != torch.float32):
        raise ValueError("s0 must be float32 (B, Hv, Dk, Dv)")
    if lengths is not None and (lengths.shape != (B,) or lengths.dtype != torch.int32):
        raise ValueError("lengths must be int32 (B,)")
    q, k, v = _rows(q), _rows(k), _rows(v)
    lds = [t.stride(1) if L > 1 else 0 for t in (q, k, v)]
    desc = GDRDesc(B, L, Hk, Hv, Dk, Dv, *lds, io=_dtype_code(v), scale=Dk ** -0.5 if scale is None else scale)
    return (desc, q, k, v, g.contiguous(), beta.contiguous(), None if s0 is None else s0.contiguous(),
            None if lengths is None else lengths.contiguous())


def _forward(prepared, flags, with_state):
    desc, q, k, v, g, beta, s0, lengths = prepared
    ws = torch.empty(max(blr_gdr_workspace_bytes(desc, flags), 16), dtype=torch.uint8, device=v.device)
    o = torch.empty(v.shape, dtype=v.dtype, device=v.device)
    s_last = None
    if with_state:
        s_last = torch.empty(desc.B, desc.Hv, desc.Dk, desc.Dv, dtype=torch.float32, device=v.device)
    blr_gdr_fwd(desc, flags, lengths, q, k, v, g, beta, s0, o, s_last, ws)
    return o, s_last, ws


class GatedDeltaRule(torch.autograd.Function):
    """(o, s_last or None) with gradients for q, k, v, g, beta and s0; see gated_delta_rule."""

    @staticmethod
    def forward(ctx, q, k, v, g, beta, scale, s0, lengths, with_state):
        flags = BLR_GDR_TRAIN | (BLR_GDR_STATE if with_state or s0 is not None else 0)
        prepared = _prepare(q, k, v, g, beta, scale, s0, lengths)
        o, s_last, ws = _forward(prepared, flags, with_state)
        ctx.save_for_backward(*prepared[1:], ws)
        ctx.desc, ctx.flags = prepared[0], flags
        ctx.set_materialize_grads(False)
        return o, s_last

    @staticmethod
    def backward(ctx, do, ds_last):
        if torch.is_grad_enabled():
            raise RuntimeError("the gated delta rule has no second derivative (create_graph=True)")
        q, k, v, g, beta, s0, lengths, ws = ctx.saved_tensors
        do = torch.zeros_like(v, memory_format=torch.contiguous_format) if do is None else do.contiguous()
        ds_last = None if ds_last is None else ds_last.contiguous()
        new = lambda t: torch.empty_like(t, memory_format=torch.contiguous_format)  # noqa: E731
        dq, dk, dv, dg, dbeta = new(q), new(k), new(v), new(g), new(beta)
        ds0 = new(s0) if s0 is not None and ctx.needs_input_grad[6] else None
        blr_gdr_bwd(ctx.desc, ctx.flags, lengths, do, ds_last, q, k, v, g, beta, s0, dq, dk, dv, dg, dbeta, ds0, ws)
        return dq, dk, dv, dg, dbeta, None, ds0, None, None


def gated_delta_rule(q, k, v, g, beta, scale: Optional[float] = None, s0=None, lengths=None,
                     with_state: bool = False):
    """The gated delta rule over whole sequences, in the tensors' dtype (float32 or bfloat16).

    q, k (B, L, Hk, Dk); v (B, L, Hv, Dv); g (the decay's logarithm, <= 0) and beta (B, L, Hv);
    s0 (B, Hv, Dk, Dv) float32 or None; lengths (B) int32 or None: row b is its last lengths[b]
    steps, the left-padding's outputs and gradients are zero. scale defaults to Dk^-0.5. q, k
    and v may be slices of wider rows. Returns (o, s_last); s_last, float32, is None unless
    with_state."""
    tracked = torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (q, k, v, g, beta, s0))
    if tracked:
        return GatedDeltaRule.apply(q, k, v, g, beta, scale, s0, lengths, with_state)
    flags = BLR_GDR_STATE if with_state or s0 is not None else 0
    return _forward(_prepare(q, k, v, g, beta, scale, s0, lengths), flags, with_state)[:2]


class GatedDeltaLayer(nn.Module):
    """A recurrent layer on the gated delta rule.

        q | k | v | z = Linear(x);  q, k normalised to length 1 per head
        g    = -exp(a) softplus(Linear_g(x) + b)     per head, a and b learned
        beta = sigmoid(Linear_beta(x))
        y    = Linear(rule(q, k, v, g, beta) * SiLU(z))

    forward() runs whole sequences (with lengths: left-padded rows, as the
    recommender's batches are), step() one new behavior per row on kept states."""

    def __init__(self, d_model: int, heads: int = 2, key_heads: Optional[int] = None, d_key: int = 64,
                 d_value: int = 64, device=None, dtype=None):
        super().__init__()
        kw = dict(device=device, dtype=dtype)
        self.heads, self.key_heads, self.d_key, self.d_value = heads, key_heads or heads, d_key, d_value
        self.sizes = [self.key_heads * d_key, self.key_heads * d_key, heads * d_value, heads * d_value, heads, heads]
        self.in_proj = nn.Linear(d_model, sum(self.sizes), **kw)
        self.out_proj = nn.Linear(heads * d_value, d_model, **kw)
        self.rate = nn.Parameter(torch.zeros(heads, **kw))
        self.rate_bias = nn.Parameter(torch.full((heads,), math.log(math.expm1(0.05)), **kw))

    def _split(self, x):
        q, k, v, z, a, b = self.in_proj(x).split(self.sizes, dim=-1)
        shape = x.shape[:2]
        unit = nn.functional.normalize
        q = unit(q.reshape(*shape, self.key_heads, self.d_key), dim=-1)
        k = unit(k.reshape(*shape, self.key_heads, self.d_key), dim=-1)
        g = -torch.exp(self.rate) * nn.functional.softplus(a + self.rate_bias)
        return q, k, v.unflatten(-1, (self.heads, self.d_value)), g, torch.sigmoid(b), z

    def forward(self, x, s0=None, lengths=None, with_state: bool = False):
        """x (B, L, d_model) -> y, or (y, states) with_state."""
        q, k, v, g, beta, z = self._split(x)
        o, s = gated_delta_rule(q, k, v, g, beta, s0=s0, lengths=lengths, with_state=with_state)
        y = self.out_proj(o.flatten(-2) * nn.functional.silu(z))
        return (y, s) if with_state else y

    @torch.no_grad()
    def step(self, x, states):
        """K new behaviors per row, x (B, K, d_model); states (float32) are updated in place."""
        q, k, v, g, beta, z = self._split(x)
        v, g, beta = v.contiguous(), g.contiguous(), beta.contiguous()
        desc = GDRDesc(*x.shape[:2], self.key_heads, self.heads, self.d_key, self.d_value, io=_dtype_code(x),
                       scale=self.d_key ** -0.5)
        o = torch.empty_like(v)
        blr_gdr_steps(desc, BLR_F32, states, q.contiguous(), k.contiguous(), v, g, beta, states, o)
        return self.out_proj(o.flatten(-2) * nn.functional.silu(z))


__all__ = ["GatedDeltaRule", "GatedDeltaLayer", "gated_delta_rule"]
