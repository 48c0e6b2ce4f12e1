"""Autograd nodes: the soft codeword (Sec. 3.5) with its BCJR-STE variant, and
the linear layer that multiplies activations with it.

``BcjrQuant`` wraps the library's entry points as a ``torch.autograd.Function``:

* soft mode: forward ``bcjr_soft_codeword`` (the soft codeword at temperature
  T), backward ``bcjr_soft_codeword_vjp``;
* hard mode (BCJR-STE, Sec. "BCJR-STE variant"): forward ``viterbi_decode``
  (the hard minimum-distortion codeword), backward ``bcjr_ste_vjp``, i.e. the
  exact gradient of the temperature-T relaxation in place of an identity
  straight-through gradient.

T is a plain number read at call time (a detached schedule value, Sec. 3.5),
so it gets no gradient.  Gradients flow to the weights and, if it requires
grad, to the codebook.  Every step runs in the library's HIP kernels.

``LinearAct8`` is activation(x W^T + bias) + residual whose backward pass reads
x and z = x W^T + bias from 8-bit checkpoints (``linear.Act8``) in place of the
activations themselves: 2.1 bytes a value pair are kept instead of 4 (bf16) or
8 (fp32).  dW is taken with the checkpoint's x, the activation's derivative at
the checkpoint's z; everything else is exact up to rounding.
"""
from __future__ import annotations

import torch

from . import bcjr_soft_codeword, bcjr_soft_codeword_vjp, bcjr_ste_vjp, viterbi_decode
from .linear import Act8, act8_store, linear_act, linear_act_vjp

__all__ = ["BcjrQuant", "bcjr_quant", "LinearAct8", "linear_act8"]


def _temperature(T) -> float:
    if isinstance(T, torch.Tensor):
        if T.numel() != 1:
            raise ValueError("T must be a scalar")
        T = T.detach().item()
    return float(T)


class BcjrQuant(torch.autograd.Function):
    """w[B, L] -> codeword[B, L] (soft at T, or hard Viterbi when ``hard``)."""

    @staticmethod
    def forward(ctx, w, codebook, state_bits, k, T, hard):
        T = _temperature(T)
        w = w.contiguous()
        codebook = codebook.contiguous()
        if hard:
            _, out = viterbi_decode(w, codebook, state_bits, k)
        else:
            out, _ = bcjr_soft_codeword(w, codebook, state_bits, k, T, want_logZ=False)
        ctx.state_bits, ctx.k, ctx.T, ctx.hard = state_bits, k, T, bool(hard)
        ctx.save_for_backward(w, codebook, out if hard else None)
        return out

    @staticmethod
    def backward(ctx, grad_out):
        w, codebook, w_hard = ctx.saved_tensors
        need_w, need_c = ctx.needs_input_grad[0], ctx.needs_input_grad[1]
        if not (need_w or need_c):
            return None, None, None, None, None, None
        g = grad_out.contiguous()
        n, k, T = ctx.state_bits, ctx.k, ctx.T
        if ctx.hard:
            dW, dc = bcjr_ste_vjp(w, codebook, n, k, T, w_hard, g, want_dW=need_w,
                                  want_dCodebook=need_c)
        else:
            dW, dc = bcjr_soft_codeword_vjp(w, codebook, n, k, T, g, want_dW=need_w,
                                            want_dCodebook=need_c)
        return dW, dc, None, None, None, None


def bcjr_quant(W, codebook, state_bits: int, k: int, T, block: int = 256, hard: bool = False):
    """Quantise a float32 tensor of any shape as consecutive blocks of ``block``
    weights (row-major; ``W.numel()`` must be a multiple of ``block``) and
    return the codeword tensor of the same shape, differentiable in W and the
    codebook."""
    if W.numel() % block:
        raise ValueError(f"W.numel() = {W.numel()} is not a multiple of block = {block}")
    out = BcjrQuant.apply(W.reshape(-1, block), codebook, state_bits, k, T, hard)
    return out.reshape(W.shape)


def _note_leaves(ctx, x):
    """Refuses to capture a layer while an eager graph over the same leaves
    lives.  A leaf's gradient is accumulated on the stream that its
    accumulation node was made on; where that is the default stream, a captured
    backward pass would order it behind the capture, which ends the process.
    The node lives as long as any graph over the leaf does, so it carries the
    mark itself."""
    if not x.is_cuda:   # (linear_act refuses it)
        return
    leaves = [n for n, _ in ctx.next_functions if n is not None and n.name() == "torch::autograd::AccumulateGrad"]
    if not leaves:
        return
    if torch.cuda.is_current_stream_capturing():
        if any("linear_act8 on the default stream" in n.metadata for n in leaves):
            raise RuntimeError("linear_act8 is being captured while the result of an eager call on the same "
                               "leaves lives: drop that result first, or run it on a stream of its own")
    elif torch.cuda.current_stream(x.device).cuda_stream == 0:
        for n in leaves:
            n.metadata["linear_act8 on the default stream"] = True


class LinearAct8(torch.autograd.Function):
    """activation(x W^T + bias) + residual with 8-bit checkpoints."""

    @staticmethod
    def forward(ctx, x, W, bias, residual, activation, x8):
        _note_leaves(ctx, x)
        need_x, need_W, need_b, need_r = ctx.needs_input_grad[:4]
        need_z = activation != "none" and (need_x or need_W or need_b)
        out = linear_act(x, W, bias, residual, activation, save=need_z)
        y, z8 = out if need_z else (out, None)
        if need_W and x8 is None:
            x8 = act8_store(x)
        ctx.activation = activation
        ctx.residual_shape = residual.shape if need_r else None
        ctx.rows, ctx.cols, ctx.dtype = x.numel() // max(x.shape[-1], 1), x.shape[-1], x.dtype
        ctx.save_for_backward(W if need_x else None, *((x8.codes, x8.scales) if need_W else (None, None)),
                              *((z8.codes, z8.scales) if need_z else (None, None)))
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        need_x, need_W, need_b, need_r = ctx.needs_input_grad[:4]
        W, xc, xs, zc, zs = ctx.saved_tensors
        g = dy.contiguous()
        x8 = Act8(xc, xs, ctx.rows, ctx.dtype) if need_W else None
        z8 = Act8(zc, zs, ctx.rows, torch.float32) if zc is not None else None
        dx, dW, db = linear_act_vjp(g, x8, W, z8, ctx.activation if z8 is not None else "none",
                                    want_dx=need_x, want_dW=need_W, want_dbias=need_b)
        # (a residual [M, N] beside an x of more dimensions, or the reverse)
        return dx, dW, db, dy.reshape(ctx.residual_shape) if need_r else None, None, None


def linear_act8(x, W, bias=None, residual=None, activation="none", x8=None):
    """activation(x W^T + bias) + residual, x [..., K], W [N, K] (float32,
    bfloat16 or float16, one type for all), differentiable in all four; the
    backward pass reads x and x W^T + bias in 8 bits.  x8: the checkpoint
    act8_store(x), where several layers read the same x.  Captured into a graph
    it is refused while the result of an eager call on the default stream, with
    a leaf in common, is kept."""
    if x8 is not None:
        if not isinstance(x8, Act8):
            raise TypeError("x8 must be an Act8")
        rows = x.numel() // max(x.shape[-1], 1)
        if (x8.rows, x8.cols, x8.dtype, x8.codes.device) != (rows, x.shape[-1], x.dtype, x.device):
            raise ValueError("x8 is not a checkpoint of x: its size, type or device differs")
    if not torch.is_grad_enabled():   # nothing to keep for a backward pass
        return linear_act(x, W, bias, residual, activation)
    return LinearAct8.apply(x, W, bias, residual, activation, x8)
