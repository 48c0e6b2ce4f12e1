"""GPU checks of the quantised linear layer against 64 bits on the CPU
(linear_reference.py, which derives the bounds)."""
import numpy as np
import pytest

import paper_2605_10655_amd as P

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import linear_reference as R  # noqa: E402
from paper_2605_10655_amd import linear as Q  # noqa: E402
from paper_2605_10655_amd.autograd import bcjr_quant, linear_act8  # noqa: E402


def _say(msg):
    print(msg, flush=True)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    P.load_library()
    yield


def rand(seed, *shape, dtype=torch.float32, scale=1.0, pad=0):
    """A CPU tensor and its GPU copy with `pad` elements between rows."""
    g = torch.Generator().manual_seed(seed)
    t = (scale * torch.randn(shape, generator=g)).to(dtype)
    if pad:
        big = torch.full((*shape[:-1], shape[-1] + pad), float("nan"), dtype=dtype, device="cuda")
        big[..., :shape[-1]] = t.cuda()
        return t, big[..., :shape[-1]]
    return t, t.cuda()


def within(got, ref, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == ref.shape, what
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isfinite(got), fine), what
    off = ((got - ref).abs() - bound)[fine]
    assert off.numel() == 0 or off.max() <= 0, f"{what}: {off.max():.3g} past the bound"


# ---------------------------------------------------------------- 8-bit checkpoints
@pytest.mark.parametrize("t", R.TYPES)
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 300, 0), (31, 7, 3), (32, 64, 0), (33, 65, 1),
                                           (100, 257, 8), (70, 8, 0)])
def test_act8_equals_the_definition(t, rows, cols, pad):
    dt = R.TYPES[t]
    _say(f"[act8] {t} {rows}x{cols} pad {pad}")
    x, xd = rand(rows * cols, rows, cols, dtype=dt, pad=pad)
    x[:, 0] *= 1000
    xd[:, 0] *= 1000
    codes, scales, v = R.act8_64(x, t == "fp16")
    a = Q.act8_store(xd)
    assert torch.equal(a.codes.cpu().double(), codes) and torch.equal(a.scales.cpu().double(), scales)
    assert torch.equal(Q.act8_load(a).cpu().double(), v)
    assert a.rows == rows and a.dtype == dt and a.nbytes == codes.numel() + 2 * scales.numel()
    for other in R.TYPES.values():
        assert torch.equal(Q.act8_load(a, other).cpu(), v.float().to(other))


@pytest.mark.parametrize("t", R.TYPES)
def test_act8_of_extreme_values(t):
    dt = R.TYPES[t]
    f = torch.finfo(dt)
    x = torch.zeros(40, 9, dtype=dt)
    x[3, 0] = f.max
    x[:, 1] = -f.max
    x[5, 2] = f.tiny
    x[6, 3] = f.smallest_normal / 4 if t != "fp32" else 2.0 ** -128
    x[0, 4], x[1, 4], x[2, 4] = float("inf"), 5.0, -1.0
    x[33, 5], x[34, 5] = float("nan"), 2.0
    x[:, 6] = 127.0
    x[:, 7] = torch.arange(40) * 0.5
    x[:, 8] = float("-inf")
    _say(f"[act8 extremes] {t}")
    codes, scales, v = R.act8_64(x, t == "fp16")
    a = Q.act8_store(x.cuda())
    assert torch.equal(a.codes.cpu().double(), codes) and torch.equal(a.scales.cpu().double(), scales)
    got = Q.act8_load(a).cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(v))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(v))


def test_act8_of_nothing_and_of_three_dimensions():
    a = Q.act8_store(torch.empty(0, 5, device="cuda"))
    assert a.codes.shape == (0, 5, 32) and Q.act8_load(a).shape == (0, 5)
    x, xd = rand(3, 4, 9, 6)
    a = Q.act8_store(xd)
    assert a.rows == 36 and torch.equal(Q.act8_load(a).cpu().double(), R.act8_64(x.view(36, 6))[2])
    # the last group's missing rows are written, as zeros
    assert not a.codes[1, :, 4:].any()


# ---------------------------------------------------------------- product
SIZES = [(1, 1, 1), (1, 100, 513), (2, 8, 64), (3, 257, 100), (16, 64, 128), (17, 33, 72), (31, 130, 65), (64, 128, 256),
         (65, 200, 264), (100, 257, 96), (130, 140, 7), (257, 129, 320), (300, 520, 136)]


def _layer(seed, M, N, K, dt, pad=0, bias=True, residual=True):
    x, xd = rand(seed, M, K, dtype=dt, pad=pad)
    W, Wd = rand(seed + 1, N, K, dtype=dt, scale=K ** -0.5, pad=pad)
    b, bd = rand(seed + 2, N, dtype=dt, scale=0.3) if bias else (None, None)
    r, rd = rand(seed + 3, M, N, dtype=dt, pad=pad) if residual else (None, None)
    return (x, W, b, r), (xd, Wd, bd, rd)


def _check_linear(host, devi, act, dt, what):
    y, yb, z, zb = R.linear64(*host, act, dt)
    got, z8 = Q.linear_act(*devi, act, save=True)
    within(got, y, yb, what)
    # without the checkpoint: up to 16 tokens by another kernel, which adds the
    # K products in another order; the bound holds for any order
    plain = Q.linear_act(*devi, act)
    within(plain, y, yb, what + " without checkpoint")
    assert len(y) <= 16 or torch.equal(plain, got)
    # the checkpoint: half a step off, the step not larger than need be
    v = R.values64(z8.codes.cpu(), z8.scales.cpu(), z.shape[0])
    M, N = z.shape
    assert z8.rows == M and z8.dtype == torch.float32
    s = z8.scales.cpu().double()
    step = s.repeat_interleave(32, 0)[:M]
    within(v, z, 0.5 * step + zb, what + " z8")
    G = s.shape[0]
    zz = torch.zeros(G * 32, N, dtype=torch.float64)
    zz[:M] = z.abs() + zb
    assert (s / 2 * 127 <= zz.view(G, 32, N).amax(1).clamp(min=127 * 2.0 ** -126)).all(), what
    tail = z8.codes.cpu()[-1, :, M - 32 * (G - 1):]
    assert not tail.any(), what


@pytest.mark.parametrize("t", R.TYPES)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear_sizes(t, M, N, K):
    _say(f"[linear] {t} {M}x{N}x{K}")
    host, devi = _layer(M * 7 + N, M, N, K, R.TYPES[t])
    _check_linear(host, devi, "silu", R.TYPES[t], f"{t} {M}x{N}x{K}")


# the tiles of large products, whole ones and ragged ones, aligned and not
LARGE = [(1930, 2056, 136, 8), (1930, 2051, 75, 3), (3900, 3592, 72, 0), (3841, 3587, 70, 1)]


@pytest.mark.parametrize("t", R.TYPES)
@pytest.mark.parametrize("M,N,K,pad", LARGE)
def test_linear_large_tiles(t, M, N, K, pad):
    _say(f"[linear large] {t} {M}x{N}x{K} pad {pad}")
    host, devi = _layer(M + N, M, N, K, R.TYPES[t], pad)
    _check_linear(host, devi, "gelu_tanh", R.TYPES[t], f"{t} {M}x{N}x{K}")


@pytest.mark.parametrize("t", R.TYPES)
@pytest.mark.parametrize("act", R.ACTS)
@pytest.mark.parametrize("M,pad,bias,residual", [(1, 0, True, False), (5, 8, False, True), (70, 3, True, True),
                                                 (133, 8, False, False), (200, 16, True, True)])
def test_linear_forms(t, act, M, pad, bias, residual):
    _say(f"[linear forms] {t} {act} M={M} pad={pad}")
    host, devi = _layer(M + pad, M, 136, 192, R.TYPES[t], pad, bias, residual)
    _check_linear(host, devi, act, R.TYPES[t], f"{t} {act} M={M}")


def test_linear_of_no_tokens_and_of_three_dimensions():
    _, (x, W, b, _r) = _layer(5, 12, 24, 40, torch.float32)
    assert Q.linear_act(x[:0], W, b).shape == (0, 24)
    y, z8 = Q.linear_act(x[:0], W, b, None, "silu", save=True)
    assert y.shape == (0, 24) and z8.codes.shape == (0, 24, 32)
    y = Q.linear_act(x, W, b, None, "gelu")
    assert torch.equal(Q.linear_act(x.view(3, 4, 40), W, b, None, "gelu"), y.view(3, 4, 24))
    out = torch.empty(12, 24, device="cuda")
    assert Q.linear_act(x, W, b, None, "gelu", out=out) is out and torch.equal(out, y)


@pytest.mark.parametrize("t", R.TYPES)
@pytest.mark.parametrize("M", [1, 16])
def test_a_few_tokens_need_no_workspace(t, M, monkeypatch):
    """Neither from Python, which does not ask for its size, nor from C, where
    a product of so long a sum would have one; with a checkpoint it still does."""
    dt = R.TYPES[t]
    host, (x, W, b, r) = _layer(M, M, 72, 20000, dt)
    y, yb, _, _ = R.linear64(*host, "silu", dt)
    lib, s = Q._lib(), torch.cuda.current_stream().cuda_stream
    assert lib.qat_linear_act_workspace_bytes(Q.DTYPES[dt], M, 72, 20000) > 0
    out, z8 = torch.empty_like(r), Q._new_act8(M, 72, torch.float32, x.device)
    args = [x.data_ptr(), 20000, W.data_ptr(), 20000, b.data_ptr(), r.data_ptr(), 72, Q.DTYPES[dt], 1, M, 72, 20000,
            out.data_ptr(), 72]
    assert lib.qat_linear_act(*args, None, None, None, 0, s) == 0
    within(out, y, yb, f"{t} M={M}")
    assert lib.qat_linear_act(*args, z8.codes.data_ptr(), z8.scales.data_ptr(), None, 0, s) == -3
    monkeypatch.setattr(Q, "_linear_bytes", None)
    assert torch.equal(Q.linear_act(x, W, b, r, "silu"), out)
    with pytest.raises(TypeError):
        Q.linear_act(x, W, b, r, "silu", save=True)


@pytest.mark.parametrize("t", R.TYPES)
def test_non_finite_values_stay_in_their_rows(t):
    """A padded row's infinities and NaN reach that row's outputs alone, and
    in the checkpoint that row's codes alone."""
    dt = R.TYPES[t]
    for M in (6, 90):
        host, devi = _layer(M, M, 72, 64, dt)
        y, z8 = Q.linear_act(*devi, "silu", save=True)
        plain = Q.linear_act(*devi, "silu")
        bad = [2, M - 1]
        devi[0][2] = float("nan")
        devi[0][M - 1] = float("inf")
        got, g8 = Q.linear_act(*devi, "silu", save=True)
        keep = [i for i in range(M) if i not in bad]
        assert torch.equal(got[keep], y[keep]) and not torch.isfinite(got[2]).any()
        got = Q.linear_act(*devi, "silu")
        assert torch.equal(got[keep], plain[keep]) and not torch.isfinite(got[2]).any()
        v = R.values64(g8.codes.cpu(), g8.scales.cpu(), M)
        assert torch.isfinite(v[keep]).all() and torch.isnan(v[2]).all()
        assert (g8.scales[0] < 0).all()


def test_linear_repeats_bit_for_bit():
    for t in R.TYPES.values():
        for M in (1, 40, 300):
            _, devi = _layer(M, M, 300, 500, t)
            y = Q.linear_act(*devi, "gelu_tanh")
            for _ in range(3):
                assert torch.equal(Q.linear_act(*devi, "gelu_tanh"), y)


# ---------------------------------------------------------------- backward
def _vjp_case(seed, M, N, K, dt, act, pad=0, dense=False):
    """Reference and arguments; dense: the checkpoints' values as the GPU
    reads them back (test_act8_equals_the_definition holds them to the
    definition), which is quick for large ones."""
    x, xd = rand(seed, M, K, dtype=dt)
    W, Wd = rand(seed + 1, N, K, dtype=dt, scale=N ** -0.5, pad=pad)
    dy, dyd = rand(seed + 2, M, N, dtype=dt, scale=M ** -0.5, pad=pad)
    z, zd = rand(seed + 3, M, N, scale=2.0)
    x8, z8 = Q.act8_store(xd), Q.act8_store(zd) if act != "none" else None
    if dense:
        xv, zv = Q.act8_load(x8).cpu(), Q.act8_load(z8).cpu()
    else:
        xv, zv = R.act8_64(x, dt == torch.float16)[2], R.act8_64(z)[2]
    return R.vjp64(dy, xv, W, zv, act, dt), (dyd, x8, Wd, z8, act)


@pytest.mark.parametrize("t", R.TYPES)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_vjp_sizes(t, M, N, K):
    _say(f"[vjp] {t} {M}x{N}x{K}")
    ref, call = _vjp_case(M + 3 * N, M, N, K, R.TYPES[t], "silu")
    for got, r, b, what in zip(Q.linear_act_vjp(*call), ref[::2], ref[1::2], ("dx", "dW", "dbias")):
        within(got, r, b, f"{what} {t} {M}x{N}x{K}")


@pytest.mark.parametrize("t", R.TYPES)
@pytest.mark.parametrize("I,J,K,pad", LARGE)
def test_vjp_large_tiles(t, I, J, K, pad):
    """dx with few outputs to sum over, dW with few tokens."""
    for M, N, C in ((I, K, J), (K, I, J)):
        _say(f"[vjp large] {t} {M}x{N}x{C} pad {pad}")
        ref, call = _vjp_case(M + N, M, N, C, R.TYPES[t], "gelu", pad, dense=True)
        for got, r, b, what in zip(Q.linear_act_vjp(*call), ref[::2], ref[1::2], ("dx", "dW", "dbias")):
            within(got, r, b, f"{what} {t} {M}x{N}x{C}")


@pytest.mark.parametrize("t", R.TYPES)
@pytest.mark.parametrize("M,N,K", [(1024, 17, 33), (1025, 17, 33), (7, 1024, 40), (7, 1025, 40), (1, 1, 70000),
                                   (129, 300, 111), (64, 256, 256), (64, 256, 257), (2, 2, 3)])
def test_vjp_at_the_bounds_of_its_small_form(t, M, N, K):
    """One launch for up to 2^22 products and 1024 terms of a sum, several past
    them."""
    _say(f"[vjp bounds] {t} {M}x{N}x{K}")
    ref, call = _vjp_case(M + 3 * N, M, N, K, R.TYPES[t], "gelu_tanh", 5, dense=True)
    for got, r, b, what in zip(Q.linear_act_vjp(*call), ref[::2], ref[1::2], ("dx", "dW", "dbias")):
        within(got, r, b, f"{what} {t} {M}x{N}x{K}")


@pytest.mark.parametrize("t", R.TYPES)
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("M,N,K,pad", [(1500, 1501, 1003, 0), (2049, 2051, 517, 3), (1800, 1600, 777, 0), (1800, 777, 1600, 5),
                                       (4097, 515, 1030, 1)])
def test_large_odd_sizes(t, act, M, N, K, pad):
    """Rows of no whole 16 bytes are padded before large products, in both
    directions, with and without dz; what lies behind them does not count."""
    dt = R.TYPES[t]
    _say(f"[odd] {t} {act} {M}x{N}x{K} pad {pad}")
    host, devi = _layer(M, M, N, K, dt, pad)
    y, yb, z, zb = R.linear64(*host, act, dt)
    got, z8 = Q.linear_act(*devi, act, save=True)
    within(got, y, yb, "y")
    ref, call = _vjp_case(M + N, M, N, K, dt, act, pad, dense=act != "none")
    for got, r, b, what in zip(Q.linear_act_vjp(*call), ref[::2], ref[1::2], ("dx", "dW", "dbias")):
        within(got, r, b, f"{what} {t} {M}x{N}x{K}")


@pytest.mark.parametrize("t", R.TYPES)
@pytest.mark.parametrize("act", R.ACTS)
@pytest.mark.parametrize("M,pad", [(1, 0), (40, 3), (150, 8), (400, 1)])
def test_vjp_forms(t, act, M, pad):
    _say(f"[vjp forms] {t} {act} M={M}")
    ref, call = _vjp_case(M, M, 136, 96, R.TYPES[t], act, pad)
    full = Q.linear_act_vjp(*call)
    for got, r, b, what in zip(full, ref[::2], ref[1::2], ("dx", "dW", "dbias")):
        within(got, r, b, f"{what} {t} {act} M={M}")
    # each output by itself, without what it does not need
    dy, x8, W, z8, _ = call
    dx = Q.linear_act_vjp(dy, None, W, z8, act, want_dW=False, want_dbias=False)
    dW = Q.linear_act_vjp(dy, x8, None, z8, act, want_dx=False, want_dbias=False)
    db = Q.linear_act_vjp(dy, None, None, z8, act, want_dx=False, want_dW=False)
    assert torch.equal(dx[0], full[0]) and dx[1] is None and dx[2] is None
    assert torch.equal(dW[1], full[1]) and dW[0] is None and dW[2] is None
    assert torch.equal(db[2], full[2]) and db[0] is None and db[1] is None
    assert Q.linear_act_vjp(*call, want_dx=False, want_dW=False, want_dbias=False) == (None, None, None)


def test_vjp_of_no_tokens_gives_zeros():
    for act in ("none", "gelu"):
        z8 = Q.act8_store(torch.empty(0, 6, device="cuda"))
        dx, dW, db = Q.linear_act_vjp(torch.empty(0, 6, device="cuda"), Q.act8_store(torch.empty(0, 9, device="cuda")),
                                      torch.ones(6, 9, device="cuda"), z8, act)
        assert dx.shape == (0, 9) and dW.shape == (6, 9) and not dW.any() and not db.any()


def test_vjp_of_a_non_finite_row():
    """A NaN in x makes its column of dW NaN and nothing else; one in z its own
    row of dx, and the gradients that sum over the rows."""
    x, xd = rand(1, 70, 24)
    W, Wd = rand(2, 16, 24)
    dy, dyd = rand(3, 70, 16)
    z, zd = rand(4, 70, 16)
    clean = Q.linear_act_vjp(dyd, Q.act8_store(xd), Wd, Q.act8_store(zd), "silu")
    bad = xd.clone()
    bad[40, 5] = float("nan")
    got = Q.linear_act_vjp(dyd, Q.act8_store(bad), Wd, Q.act8_store(zd), "silu")
    assert torch.equal(got[0], clean[0]) and torch.equal(got[2], clean[2])
    assert torch.isnan(got[1][:, 5]).all()
    keep = [i for i in range(24) if i != 5]
    assert torch.equal(got[1][:, keep], clean[1][:, keep])
    bad = zd.clone()
    bad[40, 5] = float("inf")
    got = Q.linear_act_vjp(dyd, Q.act8_store(xd), Wd, Q.act8_store(bad), "silu")
    rows = [i for i in range(70) if not 32 <= i < 64]
    assert torch.equal(got[0][rows], clean[0][rows]) and torch.isnan(got[0][40]).all()
    assert torch.isfinite(got[0][[i for i in range(70) if i != 40]]).all()
    assert torch.isnan(got[1][5]).all() and torch.isnan(got[2][5])
    assert torch.isfinite(got[1][:5]).all() and torch.isfinite(got[2][:5]).all()


@pytest.mark.parametrize("t", R.TYPES)
@pytest.mark.parametrize("M,N,K", [(1000, 136, 264), (1025, 200, 96), (80, 300, 520), (1000, 1536, 1536),
                                   (49, 2048, 2056), (1040, 1504, 1200), (1100, 4096, 4096)])
def test_vjp_of_a_non_finite_first_value(t, M, N, K):
    """A bad value in x's first group, whose scale is read where runs past the
    last token are, stays in its column of dW: tiles of every size, and tokens
    that end inside a step of each."""
    dt = R.TYPES[t]
    _, xd = rand(1, M, K, dtype=dt)
    _, dyd = rand(3, M, N, dtype=dt, scale=M ** -0.5)
    _, zd = rand(4, M, N)
    z8 = Q.act8_store(zd)
    clean = Q.linear_act_vjp(dyd, Q.act8_store(xd), None, z8, "silu", want_dx=False)
    for value in (float("nan"), float("-inf")):
        bad = xd.clone()
        bad[0, 0] = value
        got = Q.linear_act_vjp(dyd, Q.act8_store(bad), None, z8, "silu", want_dx=False)
        assert torch.isnan(got[1][:, 0]).all()
        assert torch.equal(got[1][:, 1:], clean[1][:, 1:]) and torch.equal(got[2], clean[2])


@pytest.mark.parametrize("act", R.ACTS)
def test_gradients_match_differences(act):
    """linear_act8's gradients in fp32 against central differences of the
    64-bit layer.  x holds values that its checkpoint keeps exactly; z's does
    not, and moves the derivative by at most BEND times half its step."""
    M, N, K = 40, 12, 20
    g = torch.Generator().manual_seed(11)
    x = torch.randint(-120, 121, (M, K), generator=g).float() / 64
    x[0] = x[32] = 127 / 64
    W, b = torch.randn(N, K, generator=g) * 0.3, torch.randn(N, generator=g)
    r, dy = torch.randn(M, N, generator=g), torch.randn(M, N, generator=g)
    leaves = [t.cuda().requires_grad_() for t in (x, W, b, r)]
    y = linear_act8(*leaves, act)
    y.backward(dy.cuda())
    y64, yb, z64, zb = R.linear64(x, W, b, r, act, torch.float32)
    within(y, y64, yb, act)

    def f(x, W, b, r):
        return ((R.act64(x @ W.t() + b, act) + r) * dy.double()).sum()

    zz = torch.zeros(64, N, dtype=torch.float64)
    zz[:M] = z64.abs() + zb
    # a step 2^e is below 2 amax / 127
    step = (2 * zz.view(2, 32, N).amax(1) / 127).repeat_interleave(32, 0)[:M]
    off = dy.double().abs() * (0.0 if act == "none" else 1.0) * (BEND_STEP * step + R.BEND * zb + R.ACT_ERR + 1e-6)
    host = [t.double() for t in (x, W, b, r)]
    bounds = [off @ W.double().abs(), off.t() @ x.double().abs(), off.sum(0), torch.zeros(M, N)]
    for i, (leaf, h, bound) in enumerate(zip(leaves, host, bounds)):
        for j in range(0, h.numel(), 7):
            e = 1e-5
            up, dn = [t.clone() for t in host], [t.clone() for t in host]
            up[i].view(-1)[j] += e
            dn[i].view(-1)[j] -= e
            d = (f(*up) - f(*dn)) / (2 * e)
            got = leaf.grad.view(-1)[j].item()
            # and the sums' own roundings, below 1e-4 of terms of size <= 3
            assert abs(got - d) <= bound.reshape(-1)[j] + 1e-4, (act, i, j, got, d.item())


BEND_STEP = 0.5 * R.BEND


# ---------------------------------------------------------------- trellis codes
CODES = [(4, 2, 1, 16), (16, 2, 1, 256), (16, 4, 2, 256), (12, 2, 1, 100), (8, 4, 2, 32), (14, 3, 1, 512),
         (16, 1, 1, 64), (5, 5, 1, 7), (16, 16, 1, 3), (6, 2, 3, 96), (9, 1, 1, 1), (16, 2, 1, 768)]


@pytest.mark.parametrize("n,k,V,block", CODES)
@pytest.mark.parametrize("B", [1, 37])
def test_pack_unpack_dense(n, k, V, block, B):
    _say(f"[pack] n={n} k={k} V={V} block={block} B={B}")
    rng = np.random.default_rng(n * 31 + block)
    st = R.legal_states(rng, B, block // V, n, k)
    sd = torch.from_numpy(st).cuda()
    packed = Q.trellis_pack(sd, n, k)
    assert torch.equal(packed.cpu(), R.pack64(st, n, k))
    assert torch.equal(Q.trellis_unpack(packed, n, k, block // V), sd)
    cb, cd = rand(n, *((1 << n,) if V == 1 else (1 << n, V)))
    s, sc = rand(5, B)
    want = cb[torch.from_numpy(st).long()].view(B, block)
    assert torch.equal(Q.trellis_dense(packed, cd, n, k, V, block).cpu(), want)
    for dt in R.TYPES.values():
        got = Q.trellis_dense(packed, cd, n, k, V, block, scales=sc, dtype=dt).cpu()
        assert torch.equal(got, (s[:, None] * want).to(dt))


@pytest.mark.parametrize("n,k,V,block,B", [(16, 2, 1, 256, 5000), (16, 4, 2, 256, 4100), (14, 3, 1, 512, 2051),
                                           (16, 1, 1, 64, 16500), (15, 2, 1, 8, 131079), (12, 4, 1, 1000, 1051),
                                           (6, 2, 1, 40, 30011), (16, 2, 1, 100, 11001)])
def test_dense_of_many_weights(n, k, V, block, B):
    """Above a million weights, where the codebook passes through LDS."""
    _say(f"[dense many] n={n} k={k} V={V} block={block} B={B}")
    st = R.legal_states(np.random.default_rng(n), B, block // V, n, k)
    packed = Q.trellis_pack(torch.from_numpy(st).cuda(), n, k)
    cb, cd = rand(n, *((1 << n,) if V == 1 else (1 << n, V)))
    s, sc = rand(5, B)
    want = cb[torch.from_numpy(st).long()].view(B, block)
    assert torch.equal(Q.trellis_dense(packed, cd, n, k, V, block).cpu(), want)
    for dt in R.TYPES.values():
        got = Q.trellis_dense(packed, cd, n, k, V, block, scales=sc, dtype=dt).cpu()
        assert torch.equal(got, (s[:, None] * want).to(dt))


def test_pack_refuses_what_is_no_path():
    st = torch.from_numpy(R.legal_states(np.random.default_rng(0), 5, 20, 8, 2)).cuda()
    Q.trellis_pack(st, 8, 2)
    for at, v in (((2, 7), int(st[2, 7]) ^ 128), ((0, 0), 256), ((4, 19), -1)):
        bad = st.clone()
        bad[at] = v
        with pytest.raises(ValueError):
            Q.trellis_pack(bad, 8, 2)
        Q.trellis_pack(bad, 8, 2, check=False)
    assert Q.trellis_pack(st[:0], 8, 2).shape == (0, 2)


@pytest.mark.parametrize("n,k,V", [(8, 2, 1), (12, 1, 1), (8, 4, 2)])
def test_packed_decode_gives_the_codewords(n, k, V):
    """viterbi_decode's states, packed, are its codewords."""
    g = torch.Generator().manual_seed(n)
    W = torch.randn(24, 64, generator=g).cuda()
    cb = torch.randn((1 << n,) if V == 1 else (1 << n, V), generator=g).cuda()
    states, hard = P.viterbi_decode(W, cb, n, k) if V == 1 else P.bcjr_vec_viterbi_decode(W, cb, n, k, V)
    assert torch.equal(Q.trellis_dense(Q.trellis_pack(states, n, k), cb, n, k, V, 64), hard)


def _coded(seed, N, K, n, k, V, block):
    rng = np.random.default_rng(seed)
    st = R.legal_states(rng, N * K // block, block // V, n, k)
    cb, cd = rand(seed, *((1 << n,) if V == 1 else (1 << n, V)))
    s, sd = rand(seed + 1, N, K // block, scale=0.2)
    W = cb[torch.from_numpy(st).long()].reshape(N, K // block, block)
    return W, s, Q.trellis_pack(torch.from_numpy(st).cuda(), n, k), cd, sd


@pytest.mark.parametrize("t", R.TYPES)
@pytest.mark.parametrize("n,k,V,block,N,nb", [
    (4, 2, 1, 16, 20, 3), (16, 2, 1, 256, 40, 2), (16, 4, 2, 256, 33, 1), (12, 2, 1, 100, 17, 3),
    (8, 4, 2, 32, 8, 5), (14, 3, 1, 512, 50, 1), (16, 1, 1, 256, 16, 4), (16, 2, 1, 768, 21, 1),
    (12, 4, 1, 256, 35, 9), (10, 2, 1, 64, 19, 8), (16, 4, 2, 512, 100, 2), (6, 3, 1, 256, 1, 3)])
@pytest.mark.parametrize("M", [1, 3, 16, 17, 64, 130])
def test_trellis_linear(t, n, k, V, block, N, nb, M):
    dt = R.TYPES[t]
    K = block * nb
    _say(f"[trellis] {t} n={n} k={k} V={V} block={block} {M}x{N}x{K}")
    W, s, packed, cd, sd = _coded(n + N, N, K, n, k, V, block)
    act = R.ACTS[(n + M) % 4]
    x, xd = rand(M, M, K, dtype=dt, pad=8 if M == 3 else 0, scale=K ** -0.5)
    b, bd = rand(7, N, dtype=dt)
    r, rd = rand(8, M, N, dtype=dt)
    # the weights: one rounding to the type, and one by their scale
    Ws = (s[:, :, None].double() * W.double()).reshape(N, K)
    y, yb, _, _ = R.linear64(x, Ws, b, r, act, dt, w_err=2.1 * R.HALF[dt])
    within(Q.trellis_linear(xd, packed, cd, n, k, V, block, scales=sd, bias=bd, residual=rd, activation=act),
           y, yb, "scaled")
    y, yb, _, _ = R.linear64(x, W.reshape(N, K), None, None, "none", dt, w_err=1.1 * R.HALF[dt])
    got = Q.trellis_linear(xd, packed, cd, n, k, V, block)
    within(got, y, yb, "plain")
    assert torch.equal(Q.trellis_linear(xd, packed.view(N, nb, -1), cd, n, k, V, block), got)


@pytest.mark.parametrize("t", R.TYPES)
@pytest.mark.parametrize("n,k,V,block,N,K", [
    (16, 2, 1, 256, 1030, 1024), (16, 4, 2, 512, 4100, 512), (16, 4, 2, 256, 2049, 1024), (15, 1, 1, 256, 520, 1024),
    (14, 3, 1, 256, 1025, 256), (9, 2, 1, 128, 1030, 1024), (11, 4, 1, 8448, 5, 8448), (7, 5, 3, 96, 11, 8256)])
@pytest.mark.parametrize("M", [1, 8, 9, 40])
def test_trellis_linear_of_many_weights(t, n, k, V, block, N, K, M):
    """More weights or longer rows than one launch takes in fp32: a table of
    the codebook in LDS, or a dense matrix first."""
    dt = R.TYPES[t]
    _say(f"[trellis many] {t} n={n} k={k} V={V} block={block} {M}x{N}x{K}")
    W, s, packed, cd, sd = _coded(n + N, N, K, n, k, V, block)
    x, xd = rand(M, M, K, dtype=dt, scale=K ** -0.5)
    Ws = (s[:, :, None].double() * W.double()).reshape(N, K)
    # the weights: one rounding to the type, and one by their scale
    y, yb, _, _ = R.linear64(x, Ws, None, None, "silu", dt, w_err=2.1 * R.HALF[dt])
    within(Q.trellis_linear(xd, packed, cd, n, k, V, block, scales=sd, activation="silu"), y, yb, "scaled")


@pytest.mark.parametrize("t", R.TYPES)
@pytest.mark.parametrize("n,k,V,block,N,nb", [(16, 2, 1, 256, 3, 32), (13, 5, 1, 7, 40, 9), (5, 1, 8, 8, 33, 65),
                                              (16, 16, 1, 3, 9, 4), (9, 3, 2, 10, 1, 1)])
@pytest.mark.parametrize("M", [1, 2, 4, 5, 16])
def test_few_weights_are_multiplied_in_fp32(t, n, k, V, block, N, nb, M):
    """No rounding of a weight to the type: the bound of fp32 sums alone."""
    dt = R.TYPES[t]
    K = block * nb
    _say(f"[trellis small] {t} n={n} k={k} V={V} block={block} {M}x{N}x{K}")
    W, s, packed, cd, sd = _coded(n + N, N, K, n, k, V, block)
    x, xd = rand(M, M, K, dtype=dt, scale=K ** -0.5, pad=M % 3)
    b, bd = rand(7, N, dtype=dt)
    r, rd = rand(8, M, N, dtype=dt)
    Ws = (s[:, :, None].double() * W.double()).reshape(N, K)
    # the product with the scale is rounded once, to fp32
    y, yb, _, _ = R.linear64(x, Ws, b, r, "gelu", dt, w_err=1.1 * R.HALF[torch.float32])
    within(Q.trellis_linear(xd, packed, cd, n, k, V, block, scales=sd, bias=bd, residual=rd, activation="gelu"),
           y, yb, "small")


def test_trellis_linear_of_no_tokens_and_of_three_dimensions():
    W, s, packed, cd, sd = _coded(3, 12, 64, 8, 2, 1, 32)
    x = torch.randn(2, 3, 64, device="cuda")
    y = Q.trellis_linear(x, packed, cd, 8, 2, 1, 32, scales=sd)
    assert y.shape == (2, 3, 12)
    assert torch.equal(Q.trellis_linear(x.view(6, 64), packed, cd, 8, 2, 1, 32, scales=sd), y.view(6, 12))
    assert Q.trellis_linear(x.view(6, 64)[:0], packed, cd, 8, 2, 1, 32).shape == (0, 12)


# ---------------------------------------------------------------- refusals
def test_refusals():
    x, W = torch.zeros(4, 64, device="cuda"), torch.zeros(6, 64, device="cuda")
    b, r = torch.zeros(6, device="cuda"), torch.zeros(4, 6, device="cuda")
    x8, z8 = Q.act8_store(x), Q.act8_store(r)
    bad = [
        lambda: Q.linear_act(x, W[:, :63]), lambda: Q.linear_act(x.t(), W), lambda: Q.linear_act(x, W, b[:5]),
        lambda: Q.linear_act(x, W, b, r[:3]), lambda: Q.linear_act(x, W, b, r.t().contiguous().t()),
        lambda: Q.linear_act(x.half(), W), lambda: Q.linear_act(x, W, b.half()), lambda: Q.linear_act(x.double(), W),
        lambda: Q.linear_act(x[:1].expand(4, 64), W), lambda: Q.linear_act(x, W, activation="relu"),
        lambda: Q.linear_act(x, W, out=torch.empty(4, 7, device="cuda")), lambda: Q.linear_act(x[0], W),
        lambda: Q.linear_act(x[:, :6], W[:, :6], None, r, out=r), lambda: Q.linear_act(x, W.view(2, 3, 64)),
        lambda: Q.linear_act(x.view(2, 2, 64).transpose(0, 1), W), lambda: Q.linear_act(x, W.cpu()),
        lambda: Q.linear_act_vjp(r, x8, W, None, "silu"), lambda: Q.linear_act_vjp(r, x8, W, x8, "silu"),
        lambda: Q.linear_act_vjp(r, z8, W), lambda: Q.linear_act_vjp(r[:3], x8, W),
        lambda: Q.linear_act_vjp(r.half(), x8, W.half()), lambda: Q.linear_act_vjp(r, None, W),
        lambda: Q.linear_act_vjp(r, Q.Act8(x8.codes, x8.scales, 40, x8.dtype), W),
        lambda: Q.linear_act_vjp(r, Q.Act8(x8.codes[:, ::2], x8.scales, 4, x8.dtype), W),
        lambda: Q.act8_load(x8, torch.float64), lambda: Q.act8_load(x), lambda: Q.act8_store(x.t()),
    ]
    cb, packed = torch.zeros(256, device="cuda"), torch.zeros(12, 3, dtype=torch.int32, device="cuda")
    ok = dict(state_bits=8, k=2, V=1, block=32)
    Q.trellis_linear(x, packed, cb, **ok)
    bad += [
        lambda: Q.trellis_linear(x[:, :48], packed, cb, **ok), lambda: Q.trellis_linear(x, packed[:11], cb, **ok),
        lambda: Q.trellis_linear(x, packed, cb[:128], **ok), lambda: Q.trellis_linear(x, packed.long(), cb, **ok),
        lambda: Q.trellis_linear(x, packed[:, :2].contiguous(), cb, **ok),
        lambda: Q.trellis_linear(x, packed, cb.half(), **ok),
        lambda: Q.trellis_linear(x, packed, cb, **ok, scales=torch.ones(11, device="cuda")),
        lambda: Q.trellis_linear(x, packed, cb, **ok, scales=torch.ones(12, device="cuda").half()),
        lambda: Q.trellis_linear(x, packed, cb, **{**ok, "state_bits": 17}),
        lambda: Q.trellis_linear(x, packed, cb, **{**ok, "V": 2}), lambda: Q.trellis_linear(x, packed[:0], cb, **ok),
        lambda: Q.trellis_dense(packed, cb, 8, 2, 1, 32, dtype=torch.float64),
        lambda: Q.trellis_unpack(packed, 8, 2, 60), lambda: Q.trellis_pack(packed[:, ::2], 8, 2),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((TypeError, ValueError)):
            call()
            print("not refused:", i, flush=True)
    # an overlapping output by a view
    big = torch.zeros(8, 64, device="cuda")
    with pytest.raises(ValueError):
        Q.linear_act(big[:4], torch.zeros(64, 64, device="cuda"), out=big[3:7])
    x = torch.zeros(17, 64, device="cuda")
    Q.trellis_linear(x, packed, cb, **ok)
    with pytest.raises(P.BcjrError):
        Q.trellis_linear(x, packed, cb, **ok, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


def test_a_codebook_out_of_line_is_refused_by_name():
    """A view that does not begin at 16 bytes; one that does is taken."""
    _, s, packed, cd, sd = _coded(5, 12, 64, 8, 2, 1, 32)
    x = torch.ones(3, 64, device="cuda")
    want = Q.trellis_linear(x, packed, cd, 8, 2, 1, 32)
    for off in (1, 2, 3, 4):
        view = torch.zeros(264, device="cuda")[off:off + 256]
        view.copy_(cd)
        if off % 4:
            for call in (lambda: Q.trellis_linear(x, packed, view, 8, 2, 1, 32),
                         lambda: Q.trellis_dense(packed, view, 8, 2, 1, 32)):
                with pytest.raises(ValueError, match="16 bytes"):
                    call()
        else:
            assert torch.equal(Q.trellis_linear(x, packed, view, 8, 2, 1, 32), want)
    a = Q.act8_store(x)
    codes = torch.zeros(a.codes.numel() + 8, dtype=torch.int8, device="cuda")[8:].view(a.codes.shape)
    with pytest.raises(ValueError, match="16 bytes"):
        Q.act8_load(Q.Act8(codes, a.scales, a.rows, a.dtype))


# ---------------------------------------------------------------- streams, graphs, autograd
def test_other_streams():
    host, devi = _layer(9, 200, 300, 500, torch.bfloat16)
    want = Q.linear_act(*devi, "silu", save=True)
    x8 = Q.act8_store(devi[0])
    grads = Q.linear_act_vjp(devi[3], x8, devi[1], want[1], "silu")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        y, z8 = Q.linear_act(*devi, "silu", save=True, stream=s)
        g = Q.linear_act_vjp(devi[3], Q.act8_store(devi[0], stream=s), devi[1], z8, "silu", stream=s)
        v = Q.act8_load(z8, stream=s)
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(y, want[0]) and torch.equal(z8.codes, want[1].codes)
        assert all(torch.equal(a, b) for a, b in zip(g, grads)) and torch.equal(v, Q.act8_load(want[1]))


def _entry_points():
    """Every entry point of the layer as a call of `stream`, at sizes whose
    products are split and whose odd operands are padded, so that they take
    workspaces."""
    _, (x, W, b, r) = _layer(4, 300, 264, 4100, torch.bfloat16)
    _, (xl, Wl, bl, rl) = _layer(5, 1500, 1501, 1003, torch.bfloat16)
    x8, xl8 = Q.act8_store(x), Q.act8_store(xl)
    z8, zl8 = (Q.linear_act(*a, None, "silu", save=True)[1] for a in ((x, W, b), (xl, Wl, bl)))
    _, s, packed, cd, sd = _coded(3, 264, 4096, 10, 2, 1, 256)
    states = Q.trellis_unpack(packed, 10, 2, 256)
    xc = x[:, :4096].contiguous()
    return {
        "act8_store": lambda s: Q.act8_store(x, stream=s),
        "act8_load": lambda s: Q.act8_load(x8, stream=s),
        "linear_act": lambda s: Q.linear_act(x, W, b, r, "silu", stream=s),
        "linear_act with a checkpoint": lambda s: Q.linear_act(x, W, b, r, "silu", save=True, stream=s),
        "linear_act, padded": lambda s: Q.linear_act(xl, Wl, bl, rl, "silu", stream=s),
        "linear_act_vjp": lambda s: Q.linear_act_vjp(r, x8, W, z8, "silu", stream=s),
        "linear_act_vjp, padded": lambda s: Q.linear_act_vjp(rl, xl8, Wl, zl8, "silu", stream=s),
        "trellis_pack": lambda s: Q.trellis_pack(states, 10, 2, check=False, stream=s),
        "trellis_unpack": lambda s: Q.trellis_unpack(packed, 10, 2, 256, stream=s),
        "trellis_dense": lambda s: Q.trellis_dense(packed, cd, 10, 2, scales=sd, stream=s),
        "trellis_linear": lambda s: Q.trellis_linear(xc, packed, cd, 10, 2, scales=sd, bias=b, stream=s),
    }


def _tensors(out):
    parts = out if isinstance(out, tuple) else (out,)
    return [t for p in parts for t in ((p.codes, p.scales) if isinstance(p, Q.Act8) else (p,))]


def test_calls_on_a_stream_allocate_from_its_pool(monkeypatch):
    """What the current stream has freed, and may still be writing, is not what
    a call on another stream gets for its outputs and its workspace."""
    calls = _entry_points()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    asked, real = [], Q._space
    monkeypatch.setattr(Q, "_space", lambda *a: asked.append(torch.cuda.current_stream()) or real(*a))
    for name, call in calls.items():
        _say(f"[pool] {name}")
        first = _tensors(call(None))
        want, freed = [t.clone() for t in first], {t.data_ptr() for t in first}
        del first
        torch.cuda.synchronize()
        asked.clear()
        got = _tensors(call(s))
        s.synchronize()
        assert not freed & {t.data_ptr() for t in got}, name
        assert all(a == s for a in asked), name
        assert all(torch.equal(a, b) for a, b in zip(got, want)), name
        assert torch.cuda.current_stream() != s


def test_the_current_and_another_stream_at_once():
    """Calls queued on the current stream behind long work, and the same on
    another stream at once: neither touches the other's workspace."""
    calls = _entry_points()
    want = {name: [t.clone() for t in _tensors(call(None))] for name, call in calls.items()}
    a = torch.randn(6144, 6144, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for name, call in calls.items():
        _say(f"[at once] {name}")
        got = []
        for _ in range(3):
            torch.mm(a, a)
            got += [_tensors(call(None)), _tensors(call(s))]
        torch.cuda.synchronize()
        for g in got:
            assert all(torch.equal(p, q) for p, q in zip(g, want[name])), name


@pytest.mark.parametrize("M", [1, 40, 300])
def test_captured_calls_replay(M):
    """A layer's calls captured into a graph: several replays with new inputs
    between eager calls of the same shapes."""
    _, (x, W, b, r) = _layer(M, M, 136, 256, torch.bfloat16)
    Wq, s, packed, cd, sd = _coded(1, 136, 256, 10, 2, 1, 256)

    def step():
        y, z8 = Q.linear_act(x, W, b, r, "silu", save=True)
        x8 = Q.act8_store(x)
        return (y, *Q.linear_act_vjp(r, x8, W, z8, "silu"), Q.act8_load(x8),
                Q.trellis_linear(x, packed, cd, 10, 2, scales=sd, bias=b, residual=r, activation="gelu"))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        out1 = step()
    with torch.cuda.graph(g2):
        out2 = step()
    for i in range(4):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(i)))
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        g1.replay()
        g2.replay()
        torch.cuda.synchronize()
        for a, c, w in zip(out1, out2, want):
            assert torch.equal(a, w) and torch.equal(c, w), i


def test_autograd_gives_the_calls_gradients():
    host, devi = _layer(21, 70, 40, 96, torch.bfloat16)
    leaves = [t.clone().requires_grad_() for t in devi]
    y = linear_act8(*leaves, "gelu")
    dy = torch.randn(70, 40, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    y.backward(dy)
    want, z8 = Q.linear_act(*devi, "gelu", save=True)
    dx, dW, db = Q.linear_act_vjp(dy, Q.act8_store(devi[0]), devi[1], z8, "gelu")
    assert torch.equal(y, want)
    for leaf, g in zip(leaves, (dx, dW, db, dy)):
        assert torch.equal(leaf.grad, g)
    # an expanded gradient, a shared checkpoint, three dimensions, some leaves frozen
    x8 = Q.act8_store(devi[0])
    x = devi[0].view(7, 10, 96).clone().requires_grad_()
    W = devi[1].clone().requires_grad_()
    linear_act8(x, W, None, None, "silu", x8=x8).sum().backward()
    one = torch.ones(70, 40, device="cuda", dtype=torch.bfloat16)
    _, z8 = Q.linear_act(devi[0], devi[1], None, None, "silu", save=True)
    dx, dW, _ = Q.linear_act_vjp(one, x8, devi[1], z8, "silu")
    assert torch.equal(x.grad.view(70, 96), dx) and torch.equal(W.grad, dW)
    for i in range(4):
        leaves = [t.clone().requires_grad_(i == j) for j, t in enumerate(devi)]
        linear_act8(*leaves, "gelu").backward(dy)
        assert all((t.grad is not None) == (i == j) for j, t in enumerate(leaves))
    with torch.no_grad():
        assert not linear_act8(*devi, "gelu").requires_grad
    with pytest.raises(ValueError):
        linear_act8(devi[0][:3], devi[1], x8=x8)


def test_gradients_of_a_residual_of_another_shape():
    _, (x, W, b, r) = _layer(3, 70, 40, 96, torch.bfloat16)
    dy = torch.randn(70, 40, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    leaves = [t.clone().requires_grad_() for t in (x, W, b, r)]
    linear_act8(*leaves, "gelu").backward(dy)
    for xs, rs in (((7, 10, 96), (70, 40)), ((70, 96), (2, 35, 40)), ((5, 14, 96), (10, 7, 40))):
        parts = [t.clone().requires_grad_() for t in (x.view(xs), W, b, r.view(rs))]
        y = linear_act8(*parts, "gelu")
        y.backward(dy.view(y.shape))
        for p, q in zip(parts, leaves):
            assert torch.equal(p.grad, q.grad.view(p.shape))


def _padded_layer():
    _, (x, W, b, r) = _layer(5, 96, 40, 64, torch.bfloat16)
    return x, W, b, r


def test_training_step_replays():
    """Forward and backward of two layers captured together, with new inputs
    between eager steps over other leaves of the same values."""
    x, W, b, r = _padded_layer()
    dy = torch.randn(96, 40, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()

    def step(x, leaves):
        h = linear_act8(x, leaves[0], leaves[1], None, "gelu")
        y = linear_act8(h, leaves[2], None, r, "silu")
        return (y, *torch.autograd.grad(y, leaves, dy))

    def leaves():
        g = torch.Generator().manual_seed(4)
        return [t.clone().requires_grad_() for t in (W, b, torch.randn(40, 40, generator=g).bfloat16().cuda())]

    static = leaves()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(x, static)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(x, static)
    for i in range(4):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(i)))
        want = [t.clone() for t in step(x, leaves())]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, w) for a, w in zip(out, want)), i


def test_capture_over_the_leaves_of_a_living_graph_is_refused(monkeypatch):
    """Without a capture: what the call asks of the stream is answered here."""
    x, W, b, r = _padded_layer()
    W, b = W.requires_grad_(), b.requires_grad_()
    y = linear_act8(x, W, b, r, "gelu")
    z = linear_act8(x, W.detach().clone().requires_grad_())
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    for leaf in (dict(bias=b), dict()):
        with pytest.raises(RuntimeError):
            linear_act8(x, W, **leaf)
    with pytest.raises(RuntimeError):
        linear_act8(x, W.detach(), b)
    linear_act8(x, W.detach(), b.detach())            # no leaf
    with torch.no_grad():
        linear_act8(x, W, b)
    kept = linear_act8(x, W.detach().clone().requires_grad_())   # another
    y.sum()
    del y
    assert linear_act8(x, W, b) is not None and kept is not None and z is not None


def test_capture_is_refused_as_long_as_the_leafs_node_lives(monkeypatch):
    """The node that accumulates a leaf's gradient outlives the result that it
    was made for while another graph over the leaf lives, on whatever stream;
    no other caller's leaves count.  (Without a capture.)"""
    x, W, b, r = _padded_layer()
    W = W.requires_grad_()
    first = linear_act8(x, W, b, r, "gelu")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = linear_act8(x, W, b, r, "gelu")
    torch.cuda.current_stream().wait_stream(side)
    del first
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(RuntimeError):
        linear_act8(x, W)
    del second
    assert linear_act8(x, W) is not None
    monkeypatch.undo()
    with torch.cuda.stream(side):
        third = linear_act8(x, W, b, r, "gelu")
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    assert linear_act8(x, W) is not None and third is not None


def test_only_leaves_count_for_a_capture(monkeypatch):
    """Another operator's node is no leaf's, whatever it keeps."""
    class Keeps(torch.autograd.Function):
        @staticmethod
        def forward(ctx, t):
            ctx.variable = 1
            return t.clone()

        @staticmethod
        def backward(ctx, g):
            return g

    x, W, _, _ = _padded_layer()
    h = Keeps.apply(W.requires_grad_())
    y = linear_act8(x, h)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    assert linear_act8(x, h) is not None and y is not None


def test_no_gradient_keeps_no_checkpoint(monkeypatch):
    x, W, b, r = _padded_layer()
    W = W.requires_grad_()
    import paper_2605_10655_amd.autograd as A
    monkeypatch.setattr(A, "act8_store", None)   # not called
    with torch.no_grad():
        assert torch.equal(linear_act8(x, W, b, r, "gelu"), Q.linear_act(x, W.detach(), b, r, "gelu"))
    with pytest.raises(TypeError):
        linear_act8(x, W, b, r, "gelu")


def test_offsets_past_32_bits():
    """70000 x 32768: every operator's last rows, which lie past 2^31 values."""
    M, N, K, last = 70000, 32768, 64, 32
    r0 = M - M % 32                                   # a group of 16 rows ends it
    g = torch.Generator().manual_seed(2)
    x, W = torch.randn(M, K, generator=g).bfloat16(), (0.1 * torch.randn(N, K, generator=g)).bfloat16()
    xd, Wd = x.cuda(), W.cuda()
    y, z8 = Q.linear_act(xd, Wd, None, None, "silu", save=True)
    want, bound, z, zb = R.linear64(x[-last:], W, None, None, "silu", torch.bfloat16)
    within(y[-last:], want, bound, "y")
    step = z8.scales[-1].cpu().double().abs()
    off = (Q.act8_load(z8, torch.float32)[r0:].cpu().double() - z[r0 - M:]).abs()
    assert bool((off <= 0.5 * step + zb[r0 - M:] * (1 + 1e-6)).all())
    del y
    # an activation of that size
    dy = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(last, N, generator=g).bfloat16()
    dy[-last:] = tail.cuda()
    a = Q.act8_store(dy)
    assert torch.equal(a.codes[-1], Q.act8_store(dy[r0:]).codes[0]) and not a.codes[:100].any()
    assert torch.equal(Q.act8_load(a)[r0:], Q.act8_load(Q.act8_store(dy[r0:])))
    del a
    # and the backward pass: all rows but the last give zeros
    x8 = Q.act8_store(xd)
    dx, dW, db = Q.linear_act_vjp(dy, x8, Wd, z8, "silu")
    xv = Q.act8_load(x8)[-last:].cpu().double()
    zv = Q.act8_load(z8, torch.float32)[-last:].cpu().double()
    ref = R.vjp64(tail, xv, W, zv, "silu", torch.bfloat16)
    # the sums have M terms, all but the last zero: no further rounding
    for got, r, b, what in ((dx[-last:], *ref[:2], "dx"), (dW, *ref[2:4], "dW"), (db, *ref[4:], "dbias")):
        within(got, r, b, what)
    assert not dx[:-last].any()


@pytest.mark.parametrize("n,k,V,N,K", [(16, 2, 1, 2048, 1024), (16, 4, 2, 1100, 1024)])
def test_captured_codes_replay(n, k, V, N, K):
    """The kernels whose tables take most of the LDS, captured."""
    W, s, packed, cd, sd = _coded(4, N, K, n, k, V, 256)
    xs = [torch.randn(M, K, device="cuda", dtype=torch.bfloat16) for M in (1, 16, 40, 100)]

    def step():
        return [Q.trellis_linear(x, packed, cd, n, k, V, scales=sd) for x in xs]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(3):
        for x in xs:
            x.normal_()
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i


def test_documented_forms():
    """Three dimensions with outputs given, shapes of codebook and scales that
    mean the same, a checkpoint read in another type."""
    g = torch.Generator().manual_seed(6)
    x, W = torch.randn(2, 9, 48, generator=g).cuda(), torch.randn(20, 48, generator=g).cuda()
    r = torch.randn(2, 9, 20, generator=g).cuda()
    out = torch.empty(2, 9, 20, device="cuda")
    y = Q.linear_act(x, W, None, r, "gelu", out=out)
    assert y is out and torch.equal(y.view(18, 20), Q.linear_act(x.view(18, 48), W, None, r.view(18, 20), "gelu"))
    dx, dW, _ = Q.linear_act_vjp(r, Q.act8_store(x), W)
    assert dx.shape == x.shape and torch.equal(dW, Q.linear_act_vjp(r.view(18, 20), Q.act8_store(x), W)[1])
    W, s, packed, cd, sd = _coded(5, 12, 64, 8, 2, 1, 32)
    want = Q.trellis_linear(x[..., :64 - 16].new_ones(3, 64), packed, cd, 8, 2, 1, 32, scales=sd)
    out = torch.empty(3, 12, device="cuda")
    got = Q.trellis_linear(torch.ones(3, 64, device="cuda"), packed.view(-1, packed.shape[-1]), cd.view(256, 1), 8, 2, 1,
                           32, scales=sd.reshape(-1), out=out)
    assert got is out and torch.equal(got, want)
    a = Q.act8_store(torch.randn(40, 6, generator=g).cuda())
    v = Q.act8_load(a)
    for t in (torch.float16, torch.bfloat16):
        assert torch.equal(Q.act8_load(a, t), v.to(t))


def test_same_tensors_twice_and_views():
    """One tensor as several operands, overlapping views as inputs, and a
    batch whose padding rows hold NaN."""
    g = torch.Generator().manual_seed(9)
    a = torch.randn(48, 48, generator=g).cuda()
    y = Q.linear_act(a, a, a[0].contiguous(), a, "silu")
    assert torch.equal(y, Q.linear_act(a.clone(), a.clone(), a[0].clone(), a.clone(), "silu"))
    x = a[:40]
    assert torch.equal(Q.linear_act(x, a[8:]), Q.linear_act(x.clone(), a[8:].clone()))
    x8 = Q.act8_store(a)
    one = Q.linear_act_vjp(a, x8, a, Q.act8_store(a), "gelu")
    two = Q.linear_act_vjp(a.clone(), Q.act8_store(a.clone()), a.clone(), Q.act8_store(a.clone()), "gelu")
    assert all(torch.equal(p, q) for p, q in zip(one, two))
    for M in (16, 17, 300):
        x, W = torch.randn(M, 64, generator=g).cuda(), torch.randn(40, 64, generator=g).cuda()
        pad = x.clone()
        pad[M - 3:] = float("nan")
        assert torch.equal(Q.linear_act(pad, W, activation="gelu_tanh")[:M - 3],
                           Q.linear_act(x, W, activation="gelu_tanh")[:M - 3])
        assert torch.isnan(Q.linear_act(pad, W)[M - 3:]).all()
    _, s, packed, cd, sd = _coded(2, 40, 256, 10, 2, 1, 256)
    x = torch.randn(16, 256, generator=g).cuda()
    pad = x.clone()
    pad[9:] = float("nan")
    assert torch.equal(Q.trellis_linear(pad, packed, cd, 10, 2, scales=sd)[:9],
                       Q.trellis_linear(x, packed, cd, 10, 2, scales=sd)[:9])


def test_two_streams_at_once():
    """The same layer on two streams, workspaces of their own."""
    _, (x, W, b, r) = _layer(6, 300, 264, 520, torch.bfloat16)
    want = Q.linear_act(x, W, b, r, "gelu", save=True)
    x8 = Q.act8_store(x)
    grads = Q.linear_act_vjp(r, x8, W, want[1], "gelu")
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(5):
        for s in streams:
            y, z8 = Q.linear_act(x, W, b, r, "gelu", save=True, stream=s)
            got.append((y, z8.codes, z8.scales, *Q.linear_act_vjp(r, x8, W, z8, "gelu", stream=s)))
    torch.cuda.synchronize()
    for y in got:
        assert all(torch.equal(p, q) for p, q in zip(y, (want[0], want[1].codes, want[1].scales, *grads)))


# ---------------------------------------------------------------- a run of them together
def test_train_then_answer():
    """A layer trained through its soft codewords, snapped, packed and asked:
    gradients at each end against 64 bits, the coded answer against the
    codewords'."""
    n, k, blk, N, K, M, T = 6, 2, 32, 24, 64, 50, 0.2
    g = torch.Generator().manual_seed(4)
    W0, c = torch.randn(N, K, generator=g), torch.randn(1 << n, generator=g)
    X, b = torch.randn(M, K, generator=g), torch.randn(N, generator=g)
    dy = torch.randn(M, N, generator=g)
    W, Xd, bd = W0.cuda().requires_grad_(), X.cuda(), b.cuda()
    soft = bcjr_quant(W, c.cuda(), n, k, T, block=blk)
    soft.retain_grad()
    y = linear_act8(Xd, soft, bd, None, "silu")
    y.backward(dy.cuda())
    host = soft.detach().cpu()
    y64, yb, z64, zb = R.linear64(X, host, b, None, "silu", torch.float32)
    within(y, y64, yb, "soft output")
    _, z8 = Q.linear_act(Xd, soft.detach(), bd, None, "silu", save=True)
    ref = R.vjp64(dy, R.act8_64(X)[2], host, R.values64(z8.codes.cpu(), z8.scales.cpu(), M), "silu", torch.float32)
    within(soft.grad, ref[2], ref[3], "gradient of the codewords")
    dW, _ = P.bcjr_soft_codeword_vjp(W.detach().view(-1, blk), c.cuda(), n, k, T, soft.grad.view(-1, blk),
                                     want_dCodebook=False)   # as the autograd node calls it
    assert torch.equal(W.grad, dW.view(N, K))
    states, hard = P.viterbi_decode(W.detach().view(-1, blk), c.cuda(), n, k)
    packed = Q.trellis_pack(states, n, k).view(N, K // blk, -1)
    ans = Q.trellis_linear(Xd, packed, c.cuda(), n, k, 1, blk, bias=bd, activation="silu")
    y64, yb, _, _ = R.linear64(X, hard.view(N, K).cpu(), b, None, "silu", torch.float32)
    within(ans, y64, yb, "coded answer")


@pytest.mark.parametrize("t,V", [("fp32", 1), ("bf16", 1), ("fp32", 2)])
def test_anneal_on_layer_outputs(t, V):
    """anneal_qat on a layer's outputs: its first loss and the final one from
    the packed codes against 64 bits."""
    from paper_2605_10655_amd.qat import QATConfig, anneal_qat
    dt = R.TYPES[t]
    n, k = (6, 2) if V == 1 else (8, 4)
    g = torch.Generator().manual_seed(8)
    W = torch.randn(16, 128, generator=g).cuda()
    c = torch.randn((1 << n,) if V == 1 else (1 << n, V), generator=g).cuda()
    X = (torch.randn(80, 128, generator=g) / 11).to(dt).cuda()
    b = torch.randn(16, generator=g).to(dt).cuda()
    cfg = QATConfig(state_bits=n, k=k, V=V, block=64, steps=3, T0=0.2, T_end=0.05)
    res = anneal_qat(W, c, cfg, X=X, bias=b, activation="silu")

    def loss64(Wh):
        W64, H64 = W.to(dt).cpu(), Wh.to(dt).cpu()
        a, ab, _, _ = R.linear64(X.cpu(), W64, b.cpu(), None, "silu", dt)
        h, hb, _, _ = R.linear64(X.cpu(), H64, b.cpu(), None, "silu", dt)
        d, e = (h - a).abs(), ab + hb
        return float((d * d).sum()) / 80, float((e * (2 * d + e)).sum()) / 80

    def close(got, ref):
        assert abs(got - ref[0]) <= ref[1] + 1e-5 * ref[0], (got, ref)   # and 1280 fp32 terms' sum

    if V == 1:
        soft = P.bcjr_soft_codeword(W.view(-1, 64), c, n, k, 0.2)[0].view_as(W)
    else:
        soft = P.bcjr_vec_soft_codeword(W.view(-1, 64), c, n, k, V, 0.2)[0].view_as(W)
    close(res.losses[0], loss64(soft))
    close(res.loss_hard, loss64(res.W_hard))
    assert res.packed.shape == (16, 2, Q.trellis_words(n, k, V, 64))
    assert torch.equal(Q.trellis_dense(res.packed, c, n, k, V, 64).view_as(W), res.W_hard)
    assert torch.isfinite(res.W).all() and res.max_drift > 0
    other = torch.cuda.Stream()
    again = anneal_qat(W, c, cfg, X=X, bias=b, activation="silu", stream=other)
    assert torch.equal(again.W, res.W) and again.losses == res.losses


def test_layer_loss_without_activation_is_the_hessians():
    """With no activation and H = X^T X / n the two losses are the same number."""
    from paper_2605_10655_amd.qat import QATConfig, anneal_qat
    g = torch.Generator().manual_seed(3)
    W, c, X = torch.randn(8, 64, generator=g), torch.randn(64, generator=g), torch.randn(200, 64, generator=g)
    cfg = QATConfig(state_bits=6, k=2, block=32, steps=2, T0=0.3, T_end=0.1)
    a = anneal_qat(W.cuda(), c.cuda(), cfg, X=X.cuda())
    H = (X.double().t() @ X.double() / 200).float().cuda()
    h = anneal_qat(W.cuda(), c.cuda(), cfg, H=H)
    # 200 x 64-term fp32 sums against 64 x 64-term ones: below 1e-4 of the loss
    assert abs(a.losses[0] - h.losses[0]) <= 1e-4 * h.losses[0]
    assert a.loss_ptq == pytest.approx(h.loss_ptq, rel=1e-4)
