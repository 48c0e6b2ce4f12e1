"""The quantised linear layer: what trains and answers with the codewords.

``linear_act`` is the product with bias, activation and residual in its
epilogue, ``act8_store`` and ``act8_load`` keep activations in 8 bits,
``linear_act_vjp`` is the product's backward pass from such checkpoints, and
``trellis_linear`` is the product with the weights held as the bit strings of
their trellis paths (``trellis_pack``), for one token as for a prompt.

    act8_store(x)                                               -> Act8
    act8_load(a)                                                -> [rows, cols]
    linear_act(x, W, bias, residual, activation)                -> y, or (y, Act8 of z) with save
    linear_act_vjp(dy, x8, W, z8, activation)                   -> (dx, dW, dbias)
    trellis_pack(states, state_bits, k)                         -> packed
    trellis_unpack(packed, state_bits, k, steps)                -> states
    trellis_dense(packed, codebook, state_bits, k, V, block)    -> W
    trellis_linear(x, packed, codebook, state_bits, k, V, block) -> y

This module checks arguments, allocates outputs and workspaces and passes
device pointers to the library's C ABI; every step runs in its HIP kernels.
Tensors are float32, bfloat16 or float16, the same for every operand of a
call. Matrices may have a row stride (columns contiguous, rows not
overlapping); x, residual and dy may have more than two dimensions if they are
contiguous. A codebook (float32) and an Act8's codes are aligned to 16 bytes,
everything else to its element. Calls run on the tensors' device, on its
current stream or `stream`; outputs and workspaces come from PyTorch's
allocator, from the pool of the stream that the call runs on, so that no two
streams share a workspace and calls captured into a graph own theirs. On
`stream` the inputs have to be ready, and live until it is done; what comes
back may be used on the current stream once that has waited for `stream`. No
call here records a graph for autograd: that is ``autograd.linear_act8``.
"""
from __future__ import annotations

import contextlib
import ctypes
import dataclasses
import functools
import math
import operator

import torch

from . import _check_ws, _keep_alive, _raise, load_library

__all__ = ["ACTIVATIONS", "Act8", "act8_store", "act8_load", "linear_act", "linear_act_vjp",
           "trellis_words", "trellis_pack", "trellis_unpack", "trellis_dense", "trellis_linear"]

ACTIVATIONS = {"none": 0, "silu": 1, "gelu": 2, "gelu_tanh": 3}
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
GROUP = 32   # rows (tokens) of an 8-bit group
FEW = 16     # tokens whose product needs no workspace unless it keeps a checkpoint


def _lib():
    L = load_library()
    if not getattr(L, "_linear_bound", False):
        vp, i64, ci, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t
        L.qat_act8_store.argtypes = [vp, ci, i64, i64, i64, vp, vp, vp]
        L.qat_act8_load.argtypes = [vp, vp, i64, i64, vp, ci, i64, vp]
        L.qat_linear_act_workspace_bytes.argtypes = [ci, i64, i64, i64]
        L.qat_linear_act.argtypes = [vp, i64, vp, i64, vp, vp, i64, ci, ci, i64, i64, i64, vp, i64, vp,
                                     vp, vp, sz, vp]
        L.qat_linear_act_vjp_workspace_bytes.argtypes = [ci, i64, i64, i64, ci]
        L.qat_linear_act_vjp.argtypes = [vp, i64, vp, vp, vp, i64, vp, vp, ci, ci, i64, i64, i64, vp, vp,
                                         vp, vp, sz, vp]
        L.trellis_words.argtypes = [ci, ci, ci, i64]
        L.trellis_words.restype = i64
        L.trellis_pack.argtypes = [vp, i64, i64, ci, ci, vp, vp, vp]
        L.trellis_unpack.argtypes = [vp, i64, i64, ci, ci, vp, vp]
        L.trellis_dense.argtypes = [vp, i64, vp, ci, ci, ci, i64, vp, vp, ci, vp]
        L.trellis_linear_workspace_bytes.argtypes = [ci, i64, i64, i64, ci, ci, ci, i64]
        L.trellis_linear.argtypes = [vp, i64, vp, vp, ci, ci, ci, i64, vp, vp, vp, i64, ci, ci, i64, i64,
                                     i64, vp, i64, vp, sz, vp]
        for f in (L.qat_linear_act_workspace_bytes, L.qat_linear_act_vjp_workspace_bytes,
                  L.trellis_linear_workspace_bytes):
            f.restype = sz
        L._linear_bound = True
    return L


# ---------------------------------------------------------------- checks
def _activation(name):
    if name not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}, got {name!r}")
    return ACTIVATIONS[name]


def _ptr(t):
    return None if t is None else t.data_ptr()


def _tensor(name, t, dtype=None, device=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if dtype is None:
        if t.dtype not in DTYPES:
            raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    elif t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, the call's tensors on {device}")


def _matrix(name, t, dtype=None, device=None, rows=None, cols=None):
    """(t as [rows, cols], its row stride): columns contiguous, rows not
    overlapping; more dimensions only if contiguous."""
    _tensor(name, t, dtype, device)
    shape = t.shape
    if len(shape) != 2:
        if len(shape) < 2:
            raise ValueError(f"{name} must have at least two dimensions, got {tuple(shape)}")
        if not t.is_contiguous():
            raise ValueError(f"{name} with more than two dimensions must be contiguous")
        t = t.view(math.prod(shape[:-1]), shape[-1])
        shape = t.shape
    n, c = shape
    if (rows is not None and n != rows) or (cols is not None and c != cols):
        raise ValueError(f"{name} must be [{'rows' if rows is None else rows}, "
                         f"{'cols' if cols is None else cols}], got {tuple(shape)}")
    ld, one = t.stride()
    if n <= 1:
        ld = c
    if (c > 1 and one != 1) or ld < c:
        raise ValueError(f"{name} must have contiguous columns and rows that do not overlap, "
                         f"got strides {t.stride()}")
    return t, max(ld, 1)


def _vector(name, t, n, dtype, device):
    if t is None:
        return
    _tensor(name, t, dtype, device)
    if tuple(t.shape) != (n,) or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous with shape ({n},), got {tuple(t.shape)}")


def _extent(t):
    lo = t.data_ptr()
    return lo, lo + (sum((s - 1) * st for s, st in zip(t.shape, t.stride())) + 1) * t.element_size()


def _apart(name, out, *inputs):
    """An output that shares memory with an input is refused: the kernels
    write parts of it while others still read."""
    if out.numel() == 0:
        return
    lo, hi = _extent(out)
    for t in inputs:
        if t is not None and t.numel():
            a, b = _extent(t)
            if a < hi and lo < b:
                raise ValueError(f"{name} overlaps an input")


def _output(name, out, shape, x, *inputs):
    """out, or a new tensor of x's type and device."""
    if out is None:
        return x.new_empty(shape)
    dtype, device = x.dtype, x.device
    _tensor(name, out, dtype, device)
    if tuple(out.shape) != tuple(shape) or not out.is_contiguous():
        raise ValueError(f"{name} must be contiguous with shape {tuple(shape)}, got {tuple(out.shape)}")
    _apart(name, out, x, *inputs)
    return out


def _space(workspace, nbytes, device):
    if workspace is not None:
        _check_ws(workspace, device)
        return workspace
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def _size(ws):
    return 0 if ws is None else ws.numel() * ws.element_size()


# Workspace sizes are arithmetic on the arguments: asked for once each.
@functools.lru_cache(maxsize=4096)
def _linear_bytes(*args):
    return int(_lib().qat_linear_act_workspace_bytes(*args))


@functools.lru_cache(maxsize=4096)
def _vjp_bytes(*args):
    return int(_lib().qat_linear_act_vjp_workspace_bytes(*args))


@functools.lru_cache(maxsize=4096)
def _trellis_bytes(*args):
    return int(_lib().trellis_linear_workspace_bytes(*args))


_HERE = contextlib.nullcontext()


def _on(stream, device):
    """The tensors' device as the current one for a call's launches, and
    `stream` as the current one for its allocations: memory freed on another
    stream, whose kernels may still use it, is not handed out to this call."""
    if stream is not None:
        if stream.device != device:
            raise ValueError(f"stream is on {stream.device}, the call's tensors on {device}")
        return torch.cuda.stream(stream)
    return _HERE if torch._C._cuda_getDevice() == device.index else torch.cuda.device(device)


def _stream(stream, device):
    """The stream's handle: the device's current stream unless one is given."""
    if stream is not None:
        return stream.cuda_stream
    return torch._C._cuda_getCurrentRawStream(device.index)


# ---------------------------------------------------------------- 8-bit checkpoints
@dataclasses.dataclass
class Act8:
    """An activation [rows, cols] in 8 bits: groups of 32 rows of one column
    with a power-of-two scale (negative where a value is not finite)."""
    codes: torch.Tensor          # int8 [ceil(rows / 32), cols, 32]
    scales: torch.Tensor         # bfloat16 [ceil(rows / 32), cols]
    rows: int
    dtype: torch.dtype           # the type whose values the codes stand for exactly

    @property
    def cols(self) -> int:
        return self.codes.shape[1]

    @property
    def nbytes(self) -> int:
        return self.codes.numel() + 2 * self.scales.numel()


def _check_act8(name, a, rows=None, cols=None, dtype=None, device=None):
    if not isinstance(a, Act8):
        raise TypeError(f"{name} must be an Act8")
    _tensor(name + ".codes", a.codes, torch.int8, device)
    _tensor(name + ".scales", a.scales, torch.bfloat16, a.codes.device)
    groups = -(-a.rows // GROUP)
    if a.codes.dim() != 3 or tuple(a.codes.shape) != (groups, a.codes.shape[1], GROUP):
        raise ValueError(f"{name}.codes must be [{groups}, cols, {GROUP}], got {tuple(a.codes.shape)}")
    if tuple(a.scales.shape) != tuple(a.codes.shape[:2]):
        raise ValueError(f"{name}.scales must be {tuple(a.codes.shape[:2])}, got {tuple(a.scales.shape)}")
    if not a.codes.is_contiguous() or not a.scales.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if a.codes.data_ptr() % 16:
        raise ValueError(f"{name}.codes must be aligned to 16 bytes")
    if (rows is not None and a.rows != rows) or (cols is not None and a.cols != cols):
        raise ValueError(f"{name} must hold [{rows}, {cols}], it holds [{a.rows}, {a.cols}]")
    if dtype is not None and a.dtype != dtype:
        raise TypeError(f"{name} was stored from {a.dtype}, the call's type is {dtype}")


def _new_act8(rows, cols, dtype, device):
    g = -(-rows // GROUP)
    return Act8(torch.empty((g, cols, GROUP), dtype=torch.int8, device=device),
                torch.empty((g, cols), dtype=torch.bfloat16, device=device), rows, dtype)


def act8_store(x, *, stream=None) -> Act8:
    """The 8-bit checkpoint of x [..., cols]: 1.0625 bytes a value, each at
    most half a step off, a step being at most 1/63.5 of its group's largest
    magnitude.  (Magnitudes past 65024 in float16, past 63.5 * 2^122 in the other
    types, are less than a step off.)"""
    lib = _lib()
    m, ld = _matrix("x", x)
    dev = m.device
    with _on(stream, dev):
        a = _new_act8(m.shape[0], m.shape[1], m.dtype, dev)
        rc = lib.qat_act8_store(_ptr(m), DTYPES[m.dtype], m.shape[0], m.shape[1], ld, _ptr(a.codes),
                                _ptr(a.scales), _stream(stream, dev))
        _raise("qat_act8_store", rc)
    _keep_alive(stream, a.codes, a.scales)
    return a


def act8_load(a: Act8, dtype=None, *, out=None, stream=None):
    """The values [rows, cols] that a checkpoint stands for, in dtype (default:
    the type it was stored from, in which they are exact)."""
    lib = _lib()
    _check_act8("a", a)
    dtype = a.dtype if dtype is None else dtype
    if dtype not in DTYPES:
        raise TypeError(f"dtype must be float32, bfloat16 or float16, got {dtype}")
    dev = a.codes.device
    with _on(stream, dev):
        if out is None:
            out = torch.empty((a.rows, a.cols), dtype=dtype, device=dev)
        else:
            _tensor("out", out, dtype, dev)
            if tuple(out.shape) != (a.rows, a.cols) or not out.is_contiguous():
                raise ValueError(f"out must be contiguous with shape {(a.rows, a.cols)}, got {tuple(out.shape)}")
            _apart("out", out, a.codes, a.scales)
        rc = lib.qat_act8_load(_ptr(a.codes), _ptr(a.scales), a.rows, a.cols, _ptr(out), DTYPES[dtype],
                               a.cols, _stream(stream, dev))
        _raise("qat_act8_load", rc)
    _keep_alive(stream, out)
    return out


# ---------------------------------------------------------------- product
def linear_act(x, W, bias=None, residual=None, activation="none", *, out=None, save=False,
               workspace=None, stream=None):
    """y = activation(x W^T + bias) + residual for x [..., K], W [N, K]: y
    [..., N].  With save also the 8-bit checkpoint of z = x W^T + bias, the
    backward pass's input: (y, Act8)."""
    lib = _lib()
    act = _activation(activation)
    m, ldx = _matrix("x", x)
    dev, t = m.device, m.dtype
    M, K = m.shape
    w, ldw = _matrix("W", W, t, dev, cols=K)
    if w is not W:
        raise ValueError(f"W must be [N, K], got {tuple(W.shape)}")
    N = w.shape[0]
    _vector("bias", bias, N, t, dev)
    res, ldr = (None, 0) if residual is None else _matrix("residual", residual, t, dev, M, N)
    with _on(stream, dev):
        y = _output("out", out, (*x.shape[:-1], N), m, w, bias, res)
        z8 = _new_act8(M, N, torch.float32, dev) if save else None
        ws = _space(workspace, 0 if M <= FEW and not save else _linear_bytes(DTYPES[t], M, N, K), dev)
        rc = lib.qat_linear_act(_ptr(m), ldx, _ptr(w), ldw, _ptr(bias), _ptr(res), ldr, DTYPES[t], act, M,
                                N, K, _ptr(y), N, _ptr(z8.codes) if save else None,
                                _ptr(z8.scales) if save else None, _ptr(ws), _size(ws), _stream(stream, dev))
        _raise("qat_linear_act", rc)
    _keep_alive(stream, y, ws, *((z8.codes, z8.scales) if save else ()))
    return (y, z8) if save else y


def linear_act_vjp(dy, x8, W, z8=None, activation="none", *, want_dx=True, want_dW=True,
                   want_dbias=True, workspace=None, stream=None):
    """Backward pass of linear_act from the checkpoints x8 = act8_store(x) and
    z8: (dx [..., K], dW [N, K], dbias [N]), None where unwanted.  W is needed
    for dx only, x8 for dW only, z8 for an activation only; the residual's
    gradient is dy.  dz = dy * activation'(z) is rounded to the tensors' type, as
    the products' operand (except in small layers); with float32 tensors it is
    not."""
    lib = _lib()
    act = _activation(activation)
    d, ldd = _matrix("dy", dy)
    dev, t = d.device, d.dtype
    M, N = d.shape
    if not (want_dx or want_dW or want_dbias):
        return None, None, None
    K, w, ldw = 1, None, 1
    if want_dx:
        w, ldw = _matrix("W", W, t, dev, rows=N)
        if w is not W:
            raise ValueError(f"W must be [N, K], got {tuple(W.shape)}")
        K = w.shape[1]
    if want_dW:
        _check_act8("x8", x8, M, K if want_dx else None, t, dev)
        K = x8.cols
    if act:
        if z8 is None:
            raise ValueError(f"activation {activation!r} needs z8")
        _check_act8("z8", z8, M, N, torch.float32, dev)
    with _on(stream, dev):
        dx = d.new_empty((*dy.shape[:-1], K)) if want_dx else None
        dW = d.new_empty((N, K)) if want_dW else None
        db = d.new_empty(N) if want_dbias else None
        ws = _space(workspace, _vjp_bytes(DTYPES[t], M, N, K, act), dev)
        rc = lib.qat_linear_act_vjp(_ptr(d), ldd, _ptr(x8.codes) if want_dW else None,
                                    _ptr(x8.scales) if want_dW else None, _ptr(w), ldw,
                                    _ptr(z8.codes) if act else None, _ptr(z8.scales) if act else None,
                                    DTYPES[t], act, M, N, K, _ptr(dx), _ptr(dW), _ptr(db), _ptr(ws),
                                    _size(ws), _stream(stream, dev))
        _raise("qat_linear_act_vjp", rc)
    _keep_alive(stream, dx, dW, db, ws)
    return dx, dW, db


# ---------------------------------------------------------------- trellis codes
@functools.lru_cache(maxsize=1024, typed=True)
def _code(state_bits, k, V, block):
    state_bits, k, V, block = map(operator.index, (state_bits, k, V, block))   # whole numbers: nothing is cut off
    few = max(state_bits, k, V, block) < 1 << 31   # (C's ints would wrap)
    words = int(_lib().trellis_words(state_bits, k, V, block)) if few else 0
    if words == 0:
        raise ValueError(f"no trellis code for state_bits = {state_bits}, k = {k}, V = {V}, "
                         f"block = {block}: 1 <= k <= state_bits <= 16, 1 <= V <= 8, V divides block")
    return words


def trellis_words(state_bits: int, k: int, V: int = 1, block: int = 256) -> int:
    """32-bit words of one path of `block` weights: state_bits bits and k more
    for every further step of V weights."""
    return _code(state_bits, k, V, block)


def trellis_pack(states, state_bits: int, k: int, *, check=True, stream=None):
    """States [..., steps] int32 of paths (viterbi_decode's) as bit strings
    [..., words] int32.  With check, a state that is out of range or does not
    follow the one before is a ValueError (this waits for the device)."""
    lib = _lib()
    _tensor("states", states, torch.int32)
    if states.dim() < 1 or not states.is_contiguous():
        raise ValueError("states must be contiguous with shape [..., steps]")
    steps = states.shape[-1]
    words = _code(state_bits, k, 1, steps)
    dev = states.device
    B = math.prod(states.shape[:-1])
    with _on(stream, dev):
        packed = torch.empty((*states.shape[:-1], words), dtype=torch.int32, device=dev)
        bad = torch.empty(1, dtype=torch.int32, device=dev) if check else None
        rc = lib.trellis_pack(_ptr(states), B, steps, int(state_bits), int(k), _ptr(packed), _ptr(bad),
                              _stream(stream, dev))
        _raise("trellis_pack", rc)
        if check:
            (torch.cuda.current_stream() if stream is None else stream).synchronize()
            n = int(bad.item())
            if n:
                raise ValueError(f"{n} states are not those of a path with state_bits = {state_bits}, k = {k}")
    _keep_alive(stream, packed)
    return packed


def trellis_unpack(packed, state_bits: int, k: int, steps: int, *, stream=None):
    """States [..., steps] int32 of bit strings [..., words]."""
    lib = _lib()
    _tensor("packed", packed, torch.int32)
    words = _code(state_bits, k, 1, steps)
    if packed.dim() < 1 or packed.shape[-1] != words or not packed.is_contiguous():
        raise ValueError(f"packed must be contiguous with shape [..., {words}], got {tuple(packed.shape)}")
    dev = packed.device
    with _on(stream, dev):
        states = torch.empty((*packed.shape[:-1], steps), dtype=torch.int32, device=dev)
        rc = lib.trellis_unpack(_ptr(packed), math.prod(packed.shape[:-1]), steps, int(state_bits), int(k),
                                _ptr(states), _stream(stream, dev))
        _raise("trellis_unpack", rc)
    _keep_alive(stream, states)
    return states


def _packed(packed, codebook, scales, state_bits, k, V, block, device=None):
    """Paths of a packed matrix, after checking it, its codebook and scales."""
    words = _code(state_bits, k, V, block)
    _tensor("packed", packed, torch.int32, device)
    if packed.dim() < 2 or packed.shape[-1] != words or not packed.is_contiguous():
        raise ValueError(f"packed must be contiguous with shape [..., {words}], got {tuple(packed.shape)}")
    dev = packed.device
    _tensor("codebook", codebook, torch.float32, dev)
    S = 1 << state_bits
    if tuple(codebook.shape) not in (((S,), (S, 1)) if V == 1 else ((S, V),)) or not codebook.is_contiguous():
        raise ValueError(f"codebook must be contiguous with {S} x {V} values, got {tuple(codebook.shape)}")
    if codebook.data_ptr() % 16:
        raise ValueError("codebook must be aligned to 16 bytes: this view of a larger tensor is not, copy it")
    B = math.prod(packed.shape[:-1])
    if scales is not None:
        _tensor("scales", scales, torch.float32, dev)
        if scales.numel() != B or not scales.is_contiguous():
            raise ValueError(f"scales must be contiguous with one value for each of the {B} paths, got "
                             f"{tuple(scales.shape)}")
    return B


def trellis_dense(packed, codebook, state_bits: int, k: int, V: int = 1, block: int = 256, *, scales=None,
                  dtype=torch.float32, stream=None):
    """The weights [B, block] of B paths [..., words]: scales[b] *
    codebook[state], rounded once to dtype."""
    lib = _lib()
    if dtype not in DTYPES:
        raise TypeError(f"dtype must be float32, bfloat16 or float16, got {dtype}")
    B = _packed(packed, codebook, scales, state_bits, k, V, block)
    dev = packed.device
    with _on(stream, dev):
        W = torch.empty((B, block), dtype=dtype, device=dev)
        rc = lib.trellis_dense(_ptr(packed), B, _ptr(codebook), int(state_bits), int(k), int(V), int(block),
                               _ptr(scales), _ptr(W), DTYPES[dtype], _stream(stream, dev))
        _raise("trellis_dense", rc)
    _keep_alive(stream, W)
    return W


def trellis_linear(x, packed, codebook, state_bits: int, k: int, V: int = 1, block: int = 256, *,
                   scales=None, bias=None, residual=None, activation="none", out=None, workspace=None,
                   stream=None):
    """y = activation(x W^T + bias) + residual for x [..., K] and W [N, K]
    given by its paths: packed [..., words] with N K / block paths, row n's
    blocks one after another, times scales (one a path) if given.  K must be a
    multiple of block.  Weights are rounded to x's type, as the product's
    operands, before or after their scale (of up to 16 tokens and few weights
    they are not); with x in float32 they stay as they are."""
    lib = _lib()
    act = _activation(activation)
    m, ldx = _matrix("x", x)
    dev, t = m.device, m.dtype
    M, K = m.shape
    B = _packed(packed, codebook, scales, state_bits, k, V, block, dev)
    if K < 1 or K % block or B % (K // block) or B == 0:
        raise ValueError(f"{B} paths of {block} weights do not make rows of {K}")
    N = B // (K // block)
    _vector("bias", bias, N, t, dev)
    res, ldr = (None, 0) if residual is None else _matrix("residual", residual, t, dev, M, N)
    with _on(stream, dev):
        y = _output("out", out, (*x.shape[:-1], N), m, packed, codebook, scales, bias, res)
        ws = _space(workspace, _trellis_bytes(DTYPES[t], M, N, K, int(state_bits), int(k), int(V),
                                              int(block)), dev)
        rc = lib.trellis_linear(_ptr(m), ldx, _ptr(packed), _ptr(codebook), int(state_bits), int(k), int(V),
                                int(block), _ptr(scales), _ptr(bias), _ptr(res), ldr, DTYPES[t], act, M, N, K,
                                _ptr(y), N, _ptr(ws), _size(ws), _stream(stream, dev))
        _raise("trellis_linear", rc)
    _keep_alive(stream, y, ws)
    return y
