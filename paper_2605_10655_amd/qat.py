"""Annealed quantisation-aware training of one weight matrix.

The loop of the paper's Algorithm "BCJR-QAT" (Sec. 3.7) for one layer, with
the exponential temperature schedule of Sec. 3.6 (Eq. anneal): at every step
the soft codeword of the current pre-image W is taken at temperature T_t,
a reconstruction loss is evaluated on it, its gradient is pulled back
through the soft codeword by the library's VJP, and an optimiser step moves
W.  At the end W is snapped to its Viterbi codeword.

Options beyond the paper's runs, each named there:
  * codebook learning: the VJP's dCodebook also moves the codebook (the
    paper's limitations section notes the relaxation admits it);
  * BCJR-STE: the forward value is the Viterbi codeword and the backward
    pass the temperature-T VJP (Sec. "BCJR-STE variant");
  * the drift-budget feasibility check of the paper's appendix: the
    expected nearest-codeword distance r = sigma_w / sqrt(2 pi S) against
    the largest drift lr * N * g_max that clipped gradient steps allow.

The loss is ||W_hat - W_target||_F^2, or with a proxy Hessian H = X^T X / n
of layer inputs X the layer-output error tr((W_hat - W_t) H (W_hat - W_t)^T).
With the inputs X [n, cols] themselves it is the output error of the whole
layer, ||f(X W_hat^T + b) - f(X W_t^T + b)||^2 / n, activation included: X is
kept in 8 bits for the gradient (linear.Act8), and the final codeword is
evaluated from its packed codes.
Every trellis computation, every product of the layer and every optimiser
update runs in the library's HIP kernels; the loss residual and the product
with H are plain tensor operations on the device.
"""
from __future__ import annotations

import dataclasses
import math

import torch

from . import (bcjr_soft_codeword, bcjr_soft_codeword_vjp, bcjr_ste_vjp, bcjr_vec_soft_codeword,
               bcjr_vec_soft_codeword_vjp, bcjr_vec_viterbi_decode, qat_adam_step, qat_sgd_step,
               viterbi_decode)
from .linear import act8_store, linear_act, linear_act_vjp, trellis_linear, trellis_pack

__all__ = ["QATConfig", "QATResult", "anneal_temperatures", "drift_budget", "anneal_qat"]


def anneal_temperatures(T0: float, T_end: float, steps: int):
    """T_i = T0 (T_end / T0)^(i / (steps - 1)), i = 0 .. steps - 1 (Eq. anneal,
    sampled at both ends)."""
    if steps < 1:
        raise ValueError("steps >= 1")
    if steps == 1:
        return [float(T0)]
    return [float(T0 * (T_end / T0) ** (i / (steps - 1))) for i in range(steps)]


def drift_budget(sigma_w: float, S: int, lr: float, steps: int, g_max: float) -> dict:
    """Necessary condition for leaving the initial Viterbi basin (the paper's
    drift-budget appendix): the per-element nearest-codeword distance
    r = sigma_w / sqrt(2 pi S) must be below the largest latent drift
    lr * steps * g_max reachable with gradients clipped at g_max."""
    r = sigma_w / math.sqrt(2.0 * math.pi * S)
    bound = lr * steps * g_max
    return {"r_voronoi": r, "max_drift": bound, "escape_possible": bound > r}


@dataclasses.dataclass
class QATConfig:
    state_bits: int
    k: int
    V: int = 1                   # weights per trellis step (1 or 2)
    block: int = 256             # weights per trellis block
    T0: float = 0.1
    T_end: float = 1e-3
    steps: int = 8
    lr: float = 1e-3
    grad_clip: float = 1.0       # elementwise clip of the pre-image gradient (g_max)
    optimizer: str = "adam"      # "adam" or "sgd"
    betas: tuple = (0.9, 0.999)
    eps: float = 1e-8
    learn_codebook: bool = False
    lr_codebook: float = 1e-4
    ste: bool = False


@dataclasses.dataclass
class QATResult:
    W: torch.Tensor              # final pre-image
    codebook: torch.Tensor       # final codebook
    W_hard: torch.Tensor         # Viterbi codeword of W
    temps: list
    losses: list                 # loss of each step's forward value
    loss_hard: float             # loss of W_hard
    loss_ptq: float              # loss of the Viterbi codeword of the initial W
    max_drift: float             # max |W - W_init| reached
    budget: dict                 # drift_budget() of the run's settings
    packed: torch.Tensor = None  # W_hard's paths [rows, cols / block, words] (linear.trellis_linear);
                                 # None where a block crosses rows


def _loss_and_grad(W_hat, target, H):
    R = W_hat - target
    if H is None:
        return float((R * R).sum()), 2.0 * R
    RH = R @ H
    return float((RH * R).sum()), 2.0 * RH


class _LayerLoss:
    """||f(X W_hat^T + b) - f(X W_t^T + b)||^2 / n and its gradient in W_hat."""

    def __init__(self, X, target, bias, activation, stream):
        self.X, self.bias, self.act, self.stream = X, bias, activation, stream
        self.x8 = act8_store(X, stream=stream)
        self.Y = linear_act(X, target.to(X.dtype), bias, None, activation, stream=stream).float()

    def of_output(self, Y) -> float:
        R = Y.float() - self.Y
        return float((R * R).sum()) / self.X.shape[0]

    def of(self, W) -> float:
        return self.of_output(linear_act(self.X, W.to(self.X.dtype), self.bias, None, self.act,
                                         stream=self.stream))

    def with_grad(self, W):
        z8 = None
        Wt = W.to(self.X.dtype)
        Y = linear_act(self.X, Wt, self.bias, None, self.act, save=self.act != "none", stream=self.stream)
        if self.act != "none":
            Y, z8 = Y
        R = Y.float() - self.Y
        # half of the 1 / n goes to each side, so that neither the gradient
        # nor the products leave a 16-bit type's range
        half = 1.0 / math.sqrt(self.X.shape[0])
        dW = linear_act_vjp((R * half).to(self.X.dtype), self.x8, Wt, z8, self.act, want_dx=False,
                            want_dbias=False, stream=self.stream)[1]
        return float((R * R).sum()) / self.X.shape[0], dW.float() * (2.0 * half)


def anneal_qat(W_init, codebook, cfg: QATConfig, target=None, H=None, stream=None, X=None, bias=None,
               activation="none") -> QATResult:
    """Run cfg.steps annealed steps on a [rows, cols] float32 device tensor.

    W_init is the starting pre-image (e.g. the weights themselves or a PTQ
    solution); target (default W_init) is what the codeword should
    reconstruct; H is an optional [cols, cols] proxy Hessian.  codebook is
    [S] (V = 1) or [S, V]; it is copied, and learned when
    cfg.learn_codebook.  In place of H, X [tokens, cols] (float32, bfloat16
    or float16) gives the loss on the layer's outputs, through bias [rows]
    (X's type) and activation; the products then run in X's type.
    """
    if stream is not None and stream != torch.cuda.current_stream(stream.device):
        # the loss's tensor operations go to the current stream: make it the
        # one asked for, and order it with the caller's on both sides
        here = torch.cuda.current_stream(stream.device)
        stream.wait_stream(here)
        try:
            with torch.cuda.stream(stream):
                res = anneal_qat(W_init, codebook, cfg, target, H, None, X, bias, activation)
        finally:   # a run that ends early too: the caller may then free the inputs
            here.wait_stream(stream)
        for t in (res.W, res.codebook, res.W_hard, res.packed):
            if t is not None:
                t.record_stream(here)
        return res
    n, k, V, blk = cfg.state_bits, cfg.k, cfg.V, cfg.block
    if X is None and (bias is not None or activation != "none"):
        raise ValueError("bias and activation belong to a loss on X")
    if X is not None:
        if H is not None:
            raise ValueError("give H or X, not both")
        if X.dim() != 2 or X.shape[0] < 1 or X.shape[1] != W_init.shape[-1]:
            raise ValueError(f"X must be [tokens, {W_init.shape[-1]}], got {tuple(X.shape)}")
        if W_init.shape[-1] % blk:
            raise ValueError("a loss on X needs rows that are whole blocks")
    if W_init.dim() != 2 or W_init.numel() % blk:
        raise ValueError("W_init must be [rows, cols] with rows * cols a multiple of block")
    if cfg.optimizer not in ("adam", "sgd"):
        raise ValueError("optimizer must be 'adam' or 'sgd'")
    target = W_init if target is None else target
    W = W_init.detach().clone().contiguous()
    c = codebook.detach().clone().contiguous()
    mW, vW = torch.zeros_like(W), torch.zeros_like(W)
    mc, vc = torch.zeros_like(c), torch.zeros_like(c)
    temps = anneal_temperatures(cfg.T0, cfg.T_end, cfg.steps)
    b1, b2 = cfg.betas
    layer = None if X is None else _LayerLoss(X, target, bias, activation, stream)

    def forward(Wb, T):
        if cfg.ste:
            if V == 1:
                return viterbi_decode(Wb, c, n, k, stream=stream)[1]
            return bcjr_vec_viterbi_decode(Wb, c, n, k, V, stream=stream)[1]
        if V == 1:
            return bcjr_soft_codeword(Wb, c, n, k, T, want_logZ=False, stream=stream)[0]
        return bcjr_vec_soft_codeword(Wb, c, n, k, V, T, want_logZ=False, stream=stream)[0]

    def backward(Wb, T, G, fwd):
        want_dc = cfg.learn_codebook
        if V == 1:
            if cfg.ste:
                return bcjr_ste_vjp(Wb, c, n, k, T, fwd, G, want_dCodebook=want_dc, stream=stream)
            return bcjr_soft_codeword_vjp(Wb, c, n, k, T, G, want_dCodebook=want_dc, stream=stream)
        return bcjr_vec_soft_codeword_vjp(Wb, c, n, k, V, T, G, want_dCodebook=want_dc,
                                          stream=stream)

    losses = []
    for i, T in enumerate(temps):
        Wb = W.view(-1, blk)
        fwd = forward(Wb, T)
        if layer is None:
            loss, G = _loss_and_grad(fwd.view_as(W), target, H)
        else:
            loss, G = layer.with_grad(fwd.view_as(W))
        losses.append(loss)
        dW, dc = backward(Wb, T, G.contiguous().view(-1, blk), fwd)
        if cfg.optimizer == "adam":
            qat_adam_step(W.view(-1, blk), dW, mW.view(-1, blk), vW.view(-1, blk), cfg.lr, b1, b2,
                          cfg.eps, i + 1, cfg.grad_clip, stream=stream)
            if cfg.learn_codebook:
                qat_adam_step(c, dc, mc, vc, cfg.lr_codebook, b1, b2, cfg.eps, i + 1, 0.0,
                              stream=stream)
        else:
            qat_sgd_step(W.view(-1, blk), dW, cfg.lr, cfg.grad_clip, stream=stream)
            if cfg.learn_codebook:
                qat_sgd_step(c, dc, cfg.lr_codebook, 0.0, stream=stream)

    def snap(Wm, cb):
        Wb = Wm.contiguous().view(-1, blk)
        if V == 1:
            states, hard = viterbi_decode(Wb, cb, n, k, stream=stream)
        else:
            states, hard = bcjr_vec_viterbi_decode(Wb, cb, n, k, V, stream=stream)
        return states, hard.view_as(Wm)

    states, W_hard = snap(W, c)
    packed = None
    if W.shape[1] % blk == 0:
        packed = trellis_pack(states.view(W.shape[0], W.shape[1] // blk, blk // V), n, k, check=False,
                              stream=stream)
    # the PTQ reference: the initial weights snapped with the initial codebook
    W_ptq = snap(W_init.detach(), codebook.detach().contiguous())[1]
    if layer is None:
        loss_hard = _loss_and_grad(W_hard, target, H)[0]
        loss_ptq = _loss_and_grad(W_ptq, target, H)[0]
    else:
        loss_hard = layer.of_output(trellis_linear(X, packed, c, n, k, V, blk, bias=bias,
                                                   activation=activation, stream=stream))
        loss_ptq = layer.of(W_ptq)
    sigma = float(target.float().std())
    return QATResult(W=W, codebook=c, W_hard=W_hard, temps=temps, losses=losses,
                     loss_hard=loss_hard, loss_ptq=loss_ptq,
                     max_drift=float((W - W_init).abs().max()),
                     budget=drift_budget(sigma, 1 << n, cfg.lr, cfg.steps, cfg.grad_clip),
                     packed=packed)
