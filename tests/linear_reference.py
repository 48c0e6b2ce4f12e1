"""The quantised linear layer in 64 bits on the CPU, from its definitions:
what the GPU tests compare with, and the bounds of their comparison."""
import math

import numpy as np
import torch

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
ACTS = ("none", "silu", "gelu", "gelu_tanh")

# Half a step of each type relative to the value, and its smallest step's half
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}
# An activation or its derivative in fp32: at most 16 operations on terms of
# size <= 1.2 (times |z| for the value), each off by at most a step 2^-23.
ACT_ERR = 16 * 2.0 ** -23
LIP = 1.13          # the activations' largest slope (gelu, gelu_tanh: 1.129)
BEND = 0.8          # their largest second derivative (gelu: 2 phi(0) = 0.798)


def act64(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2.0))
    if act == "gelu_tanh":
        return z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))
    return z


def slope64(z, act):
    z = z.clone().requires_grad_(True)
    return torch.autograd.grad(act64(z, act).sum(), z)[0]


def act8_64(x, fp16=False):
    """(codes [G, C, 32], scales [G, C], values [M, C]) of the 8-bit groups of
    x [M, C], by exact rational steps of float64."""
    x = x.double().numpy()
    M, C = x.shape
    G = -(-M // 32)
    low, high = (-24, 10) if fp16 else (-126, 122)
    codes, scales = np.zeros((G, C, 32)), np.zeros((G, C))
    for g in range(G):
        for c in range(C):
            v = x[32 * g:32 * g + 32, c]
            fin = np.isfinite(v)
            amax = np.abs(v[fin]).max() if fin.any() else 0.0
            e = low
            while amax > 127.0 * 2.0 ** e:
                e += 1
            top = 63 if e >= high else 127
            q = np.clip(np.rint(np.where(fin, v, 0.0) / 2.0 ** e), -top, top)
            codes[g, c, :len(v)] = np.where(fin, q, -128)
            scales[g, c] = 2.0 ** e if fin.all() else -(2.0 ** e)
    codes, scales = torch.from_numpy(codes), torch.from_numpy(scales)
    return codes, scales, values64(codes, scales, M)


def values64(codes, scales, M):
    q = codes.double()
    v = torch.where(q == -128, math.nan, q * scales.double().abs()[..., None])
    return v.transpose(1, 2).flatten(0, 1)[:M]


def linear64(x, W, bias, residual, act, dtype, w_err=0.0):
    """(y, bound of |y' - y|, z, bound of |z' - z|).  z' sums K products (for
    16-bit types exact, for fp32 half a step off) in fp32 in some order: each
    of the K additions is off by half a step of a partial sum, at most
    sum |x||W|.  w_err: relative error of W's own rounding."""
    x, W = x.double(), W.double()
    z = x @ W.t()
    s = x.abs() @ W.abs().t()
    if bias is not None:
        z = z + bias.double()
        s = s + bias.double().abs()
    zb = s * ((x.shape[1] + 3) * 2.0 ** -24 + w_err)
    y = act64(z, act)
    yb = LIP * zb + (0.0 if act == "none" else ACT_ERR * (1 + z.abs()))
    if residual is not None:
        y = y + residual.double()
        yb = yb + 2.0 ** -24 * (y.abs() + yb)
    # the result's rounding, of a value that is itself off by yb
    yb = yb + HALF[dtype] * (y.abs() + yb) + TINY[dtype]
    return y, yb, z, zb


def vjp64(dy, x, W, z, act, dtype):
    """(dx, bound, dW, bound, dbias, bound) for the checkpoint's x and z.  dz'
    is off by the derivative's error and two roundings (the product's and that
    to dtype); the sums as in linear64."""
    dy, x, W = dy.double(), x.double(), W.double()
    f = slope64(z.double(), act) if act != "none" else torch.ones_like(dy)
    dz = dy * f
    raw = (0.0 if act == "none" else ACT_ERR) * dy.abs() + 2.0 ** -24 * dz.abs()   # before its rounding
    half = 0.0 if act == "none" else HALF[dtype]
    off = raw + half * (dz.abs() + raw) + (0.0 if act == "none" else TINY[dtype])
    M, N = dz.shape

    def product(a, ao, b, terms):
        v, s = a @ b, (a.abs() + ao) @ b.abs()
        vb = ao @ b.abs() + s * (terms + 3) * 2.0 ** -24
        return v, vb + HALF[dtype] * (v.abs() + vb) + TINY[dtype]

    dx, dxb = product(dz, off, W, N)
    dW, dWb = product(dz.t(), off.t(), x, M)
    db = dz.sum(0)
    dbb = raw.sum(0) + (dz.abs() + raw).sum(0) * 36 * 2.0 ** -24
    dbb = dbb + HALF[dtype] * (db.abs() + dbb) + TINY[dtype]
    return dx, dxb, dW, dWb, db, dbb


def legal_states(rng, B, steps, n, k):
    """Random paths: the first state any, then k new bits a step."""
    s = np.zeros((B, steps), dtype=np.int64)
    s[:, 0] = rng.integers(0, 1 << n, B)
    for t in range(1, steps):
        s[:, t] = ((s[:, t - 1] << k) | rng.integers(0, 1 << k, B)) & ((1 << n) - 1)
    return s.astype(np.int32)


def pack64(states, n, k):
    """The bit strings of paths, character by character."""
    out = []
    for row in np.asarray(states):
        text = format(int(row[0]), f"0{n}b") + "".join(format(int(s) & ((1 << k) - 1), f"0{k}b") for s in row[1:])
        text += "0" * (-len(text) % 32)
        out.append([int(text[i:i + 32], 2) for i in range(0, len(text), 32)])
    return torch.from_numpy(np.array(out, dtype=np.uint32).view(np.int32))
