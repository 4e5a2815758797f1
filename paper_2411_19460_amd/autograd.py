"""torch.autograd faces of the C ABI.  `adapter_linear(...)` is a frozen projection with low-rank adapters, differentiable in its
input and in the adapters.  `ssd_scan(...)` is differentiable and keeps, between forward and
backward, only what MA-GC keeps (Sec. 3.2-3.3: the state entering every segment) -- the backward pass
calls ssd_bwd, which restores each segment from its checkpoint.  Argument marshalling only: every
step of the computation runs in libssd_magc.so."""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding


def _dense(grad):
    """What autograd hands in may be a view that begins anywhere in a larger gradient; the calls take dense tensors on 16 bytes."""
    grad = grad.contiguous()
    return grad if grad.data_ptr() % 16 == 0 else grad.clone()


class _SSDScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, dt, A, B, C, D, init_state, chunk, segment, flags, seq_reset):
        y, final, bnd = binding.ssd_fwd(x, dt, A, B, C, D, chunk, segment, init_state, flags, seq_reset=seq_reset)
        ctx.save_for_backward(x, dt, A, B, C, D, init_state if init_state is not None else x.new_empty(0),
                              bnd if bnd is not None else x.new_empty(0))
        ctx.cfg = (chunk, segment, flags, init_state is not None, bnd is not None)
        ctx.seq_reset = seq_reset
        return y, final

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dfinal):
        x, dt, A, B, C, D, init_state, bnd = ctx.saved_tensors
        chunk, segment, flags, has_init, has_bnd = ctx.cfg
        if dy is None:
            dy = torch.zeros_like(x)
        g = binding.ssd_bwd(x, dt, A, B, C, D, dy.contiguous(), chunk, segment, init_state if has_init else None,
                            dfinal.contiguous() if dfinal is not None else None, bnd if has_bnd else None, flags,
                            want_dinit=has_init and ctx.needs_input_grad[6], seq_reset=ctx.seq_reset)
        return (g["dx"], g["ddt"], g["dA"], g["dB"], g["dC"], g["dD"],
                g["dinit_state"] if has_init and ctx.needs_input_grad[6] else None, None, None, None, None)


def ssd_scan(x, dt, A, B, C, D, chunk, segment=None, init_state=None, flags=0, seq_reset=None):
    """y, final_state = ssd_scan(...): one SSD layer (Sec. 3.1, Eq. 1 in the Mamba-2 form), differentiable in
    x, dt, A, B, C, D and init_state.  `segment` is the checkpoint interval in tokens (None: the whole
    sequence is one segment).  seq_reset [Bt, L] uint8 marks the first token of every packed sequence.
    Tensors as in ssd_fwd (contiguous device tensors; dt already positive)."""
    return _SSDScan.apply(x, dt, A, B, C, D, init_state, chunk, segment, flags, seq_reset)


class _AdapterLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, a, b, scale, plan):
        f = binding.ssd_adapter_linear_fwd(x, w, a, b, scale, plan, want_hidden=ctx.needs_input_grad[2] or ctx.needs_input_grad[3])
        hidden = f["hidden"]
        ctx.save_for_backward(x, w, a, b, scale, hidden if hidden is not None else scale.new_empty(0))
        ctx.cfg = (plan, hidden is not None)
        return f["out"]

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        x, w, a, b, scale, hidden = ctx.saved_tensors
        plan, has_hidden = ctx.cfg
        dab = ctx.needs_input_grad[2] or ctx.needs_input_grad[3]
        g = binding.ssd_adapter_linear_bwd(x, w, a, b, scale, plan, _dense(dout), hidden if has_hidden else None,
                                           want_dx=ctx.needs_input_grad[0], want_dab=dab)
        return g["dx"], None, g["da"] if ctx.needs_input_grad[2] else None, g["db"] if ctx.needs_input_grad[3] else None, None, None


def adapter_linear(x, w, a, b, scale, plan):
    """x [rows, in_dim] @ w^T plus each row's low-rank adapter (see ssd_adapter_linear_fwd); differentiable in x, a and b.  w and scale
    are constants: where gradients are recorded neither may require one (w's is ssd_linear_bwd's).
    A gradient of a gradient is an error.  Autograd rounds the adapters' fp32 gradients to a's and b's bf16; ssd_adapter_linear_bwd hands
    them out as they are."""
    if torch.is_grad_enabled():
        for name, t in (("w", w), ("scale", scale)):
            if t.requires_grad:
                raise ValueError(f"{name} requires a gradient, and adapter_linear has none for it: pass {name}.detach()")
    return _AdapterLinear.apply(x, w, a, b, scale, plan)
