"""Host-side checks of the quantised linear layer: refusals, sizes, and the
64-bit reference that the GPU tests use."""
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import linear_reference as R  # noqa: E402
import paper_2605_10655_amd as P  # noqa: E402
from paper_2605_10655_amd import linear as Q  # noqa: E402

FAKE = 1 << 20          # 16-byte aligned non-null address, never dereferenced
INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(P.library_path()):
        pytest.skip("libbcjr.so not built")
    return Q._lib()


def change(args, **at):
    out = list(args)
    for k, v in at.items():
        out[int(k[1:])] = v
    return out


def test_act8_arguments(lib):
    ok = [FAKE, 1, 40, 8, 8, FAKE, FAKE, None]
    for bad in (dict(_0=None), dict(_0=FAKE + 1), dict(_1=3), dict(_1=-1), dict(_2=-1), dict(_3=0), dict(_4=7),
                dict(_5=None), dict(_5=FAKE + 8), dict(_6=None), dict(_6=FAKE + 1)):
        assert lib.qat_act8_store(*change(ok, **bad)) == INVALID, bad
    assert lib.qat_act8_store(*change(ok, _2=0, _0=None, _5=None, _6=None)) == 0
    assert lib.qat_act8_store(*change(ok, _2=1 << 31)) == UNSUPPORTED
    assert lib.qat_act8_store(*change(ok, _3=1 << 22, _4=1 << 22)) == UNSUPPORTED
    ok = [FAKE, FAKE, 40, 8, FAKE, 1, 8, None]
    for bad in (dict(_0=None), dict(_0=FAKE + 8), dict(_1=None), dict(_2=-1), dict(_3=0), dict(_4=None),
                dict(_4=FAKE + 1), dict(_5=9), dict(_6=7)):
        assert lib.qat_act8_load(*change(ok, **bad)) == INVALID, bad
    assert lib.qat_act8_load(*change(ok, _2=0)) == 0


def test_linear_act_arguments(lib):
    ws = lib.qat_linear_act_workspace_bytes
    for bad in ((5, 4, 8, 16), (1, -1, 8, 16), (1, 4, 0, 16), (1, 4, 8, 0)):
        assert ws(*bad) == 0
    # x ldx W ldw bias residual ldr dtype act M N K y ldy zc zs ws bytes stream
    ok = [FAKE, 16, FAKE, 16, None, None, 0, 1, 0, 4, 8, 16, FAKE, 8, None, None, FAKE, 1 << 40, None]
    for bad in (dict(_0=None), dict(_0=FAKE + 1), dict(_1=15), dict(_2=None), dict(_3=15), dict(_4=FAKE + 1),
                dict(_5=FAKE, _6=7), dict(_5=FAKE + 1, _6=8), dict(_7=3), dict(_8=4), dict(_8=-1), dict(_9=-1),
                dict(_10=0), dict(_11=0), dict(_12=None), dict(_13=7), dict(_14=FAKE), dict(_15=FAKE),
                dict(_14=FAKE + 8, _15=FAKE)):
        assert lib.qat_linear_act(*change(ok, **bad)) == INVALID, bad
    assert lib.qat_linear_act(*change(ok, _9=1 << 31)) == UNSUPPORTED
    assert lib.qat_linear_act(*change(ok, _10=1 << 22, _13=1 << 22)) == UNSUPPORTED
    assert lib.qat_linear_act(*change(ok, _9=0)) == 0          # no tokens


def test_vjp_arguments(lib):
    ws = lib.qat_linear_act_vjp_workspace_bytes
    assert ws(5, 4, 8, 16, 0) == 0 and ws(1, 4, 0, 16, 0) == 0 and ws(1, 4, 8, 16, 9) == 0
    assert ws(1, 2048, 8, 16, 1) >= 2048 * 8 * 2 + 64 * 8 * 4
    # dy ldd xc xs W ldw zc zs dtype act M N K dx dW dbias ws bytes stream
    ok = [FAKE, 8, FAKE, FAKE, FAKE, 16, FAKE, FAKE, 1, 1, 4, 8, 16, FAKE, FAKE, FAKE, FAKE, 1 << 40, None]
    for bad in (dict(_0=None), dict(_1=7), dict(_2=None), dict(_2=FAKE + 4), dict(_3=None), dict(_4=None),
                dict(_5=15), dict(_6=None), dict(_7=None), dict(_8=3), dict(_9=4), dict(_10=-1), dict(_11=0),
                dict(_12=0), dict(_13=FAKE + 1), dict(_14=FAKE + 1), dict(_15=FAKE + 1)):
        assert lib.qat_linear_act_vjp(*change(ok, **bad)) == INVALID, bad
    for bad in (dict(_16=None), dict(_16=FAKE + 8), dict(_17=16)):
        assert lib.qat_linear_act_vjp(*change(ok, _10=2048, **bad)) == WORKSPACE, bad
    assert lib.qat_linear_act_vjp(*change(ok, _13=None, _14=None, _15=None)) == 0
    assert lib.qat_linear_act_vjp(*change(ok, _12=1 << 22, _5=1 << 22)) == UNSUPPORTED


def test_trellis_arguments(lib):
    words = lib.trellis_words
    assert words(16, 2, 1, 256) == 17 and words(16, 4, 2, 256) == 17 and words(4, 4, 1, 1) == 1
    assert words(12, 1, 1, 1) == 1 and words(16, 16, 1, 3) == 2
    for bad in ((17, 2, 1, 256), (4, 5, 1, 16), (4, 0, 1, 16), (4, 2, 0, 16), (4, 2, 9, 18), (4, 2, 3, 16),
                (4, 2, 1, 0), (4, 2, 1, (1 << 24) + 1)):
        assert words(*bad) == 0, bad
    ok = [FAKE, 4, 16, 8, 2, FAKE, None, None]
    for bad in (dict(_0=None), dict(_0=FAKE + 2), dict(_1=-1), dict(_2=0), dict(_3=17), dict(_4=9), dict(_5=None),
                dict(_6=FAKE + 2)):
        assert lib.trellis_pack(*change(ok, **bad)) == INVALID, bad
    assert lib.trellis_pack(*change(ok, _1=1 << 40)) == UNSUPPORTED
    assert lib.trellis_pack(*change(ok, _1=0)) == 0
    ok = [FAKE, 4, 16, 8, 2, FAKE, None]
    for bad in (dict(_0=None), dict(_1=-1), dict(_2=0), dict(_3=17), dict(_5=None)):
        assert lib.trellis_unpack(*change(ok, **bad)) == INVALID, bad
    # packed B codebook n k V block scales W dtype stream
    ok = [FAKE, 4, FAKE, 8, 2, 1, 16, None, FAKE, 1, None]
    for bad in (dict(_0=None), dict(_1=-1), dict(_2=None), dict(_2=FAKE + 4), dict(_3=17), dict(_5=3),
                dict(_7=FAKE + 2), dict(_8=None), dict(_9=3)):
        assert lib.trellis_dense(*change(ok, **bad)) == INVALID, bad
    assert lib.trellis_dense(*change(ok, _1=0)) == 0
    ws = lib.trellis_linear_workspace_bytes
    assert ws(1, 4, 8, 100, 8, 2, 1, 16) == 0 and ws(1, 4, 8, 64, 17, 2, 1, 16) == 0
    # x ldx packed codebook n k V block scales bias residual ldr dtype act M N K y ldy ws bytes stream
    ok = [FAKE, 64, FAKE, FAKE, 8, 2, 1, 16, None, None, None, 0, 1, 0, 4, 8, 64, FAKE, 8, FAKE, 1 << 40, None]
    for bad in (dict(_0=None), dict(_1=63), dict(_2=None), dict(_3=FAKE + 4), dict(_4=17), dict(_5=0), dict(_6=3),
                dict(_7=24), dict(_8=FAKE + 1), dict(_9=FAKE + 1), dict(_10=FAKE, _11=7), dict(_12=3), dict(_13=4),
                dict(_14=-1), dict(_15=0), dict(_17=None), dict(_18=7)):
        assert lib.trellis_linear(*change(ok, **bad)) == INVALID, bad
    for bad in (dict(_19=None), dict(_19=FAKE + 8), dict(_20=16)):
        assert lib.trellis_linear(*change(ok, _14=17, **bad)) == WORKSPACE, bad
    assert lib.trellis_linear(*change(ok, _14=0)) == 0


def test_launches_and_strides_past_the_limits(lib):
    """Grids of 2^32 threads and rows further apart than 32-bit offsets reach."""
    top = (1 << 31) - 1
    for dtype in (0, 1, 2):
        es = 4 if dtype == 0 else 2
        wide = 64 * (1 if dtype == 0 else 2)     # columns of a workgroup of 64 threads and 32 rows
        assert lib.qat_act8_store(FAKE, dtype, top, wide, wide, FAKE, FAKE, None) == UNSUPPORTED
        assert lib.qat_act8_load(FAKE, FAKE, top, wide, FAKE, dtype, wide, None) == UNSUPPORTED
        far = (1 << 25) // es
        for ldx, ldw in ((far, 16), (16, far), (1 << 62, 16), (16, 1 << 62)):
            assert lib.qat_linear_act(FAKE, ldx, FAKE, ldw, None, None, 0, dtype, 0, 4, 8, 16, FAKE, 8, None, None,
                                      FAKE, 1 << 40, None) == UNSUPPORTED
            assert lib.qat_linear_act_vjp(FAKE, ldx, FAKE, FAKE, FAKE, ldw, None, None, dtype, 0, 4, 8, 16, FAKE,
                                          FAKE, FAKE, FAKE, 1 << 40, None) == UNSUPPORTED
        assert lib.trellis_linear(FAKE, far, FAKE, FAKE, 8, 2, 1, 16, None, None, None, 0, dtype, 0, 4, 8, 16, FAKE,
                                  8, FAKE, 1 << 40, None) == UNSUPPORTED
        # tiles of 64 rows by 256 threads
        assert lib.qat_linear_act(FAKE, 8, FAKE, 8, None, None, 0, dtype, 0, 1 << 30, 8, 8, FAKE, 8, None, None,
                                  FAKE, 1 << 40, None) == UNSUPPORTED
    assert lib.trellis_unpack(FAKE, 1 << 24, 256, 8, 2, FAKE, None) == UNSUPPORTED
    assert lib.trellis_dense(FAKE, 1 << 24, FAKE, 8, 2, 1, 256, None, FAKE, 0, None) == UNSUPPORTED


def test_small_layers_need_no_workspace(lib):
    need = lib.qat_linear_act_vjp_workspace_bytes
    assert need(1, 64, 256, 256, 1) == 0 and need(1, 64, 256, 257, 1) > 0
    assert need(1, 1024, 8, 8, 1) == 0 and need(1, 1025, 8, 8, 1) > 0 and need(1, 8, 1025, 8, 1) > 0
    need = lib.trellis_linear_workspace_bytes
    # dtype M N K state_bits k V block
    assert need(1, 16, 1024, 1024, 12, 2, 1, 128) == 0 and need(1, 17, 1024, 1024, 12, 2, 1, 128) > 0
    assert need(1, 16, 1032, 1024, 12, 2, 1, 128) > 0 and need(1, 1, 1, 16384, 12, 2, 1, 128) > 0
    assert need(1, 16, 4096, 4096, 12, 2, 1, 256) == 0 and need(1, 64, 2048, 2048, 12, 2, 1, 256) == 0
    assert need(1, 17, 4096, 4096, 12, 2, 1, 256) > 0 and need(1, 65, 256, 256, 12, 2, 1, 256) > 0


def test_a_trellis_is_given_by_whole_numbers(lib):
    assert Q.trellis_words(np.int64(16), 2, np.int32(1), 256) == 17
    for args in ((16.5, 2), (16.0, 2), (16, 2.5), (16, 2, 1.5), (16, 2, 1, 256.5), ("16", 2)):
        with pytest.raises(TypeError):
            Q.trellis_words(*args)
    for args in (((1 << 32) + 16, 2), (16, (1 << 32) + 2), (16, 2, (1 << 32) + 1), (16, 2, 1, (1 << 64) + 256), (16, -2)):
        with pytest.raises(ValueError):
            Q.trellis_words(*args)


def test_host_tensors_are_refused(lib):
    x, W = torch.zeros(4, 8), torch.zeros(6, 8)
    for call in (lambda: Q.act8_store(x), lambda: Q.linear_act(x, W), lambda: Q.linear_act_vjp(x, None, W),
                 lambda: Q.trellis_pack(torch.zeros(2, 4, dtype=torch.int32), 4, 2),
                 lambda: Q.trellis_unpack(torch.zeros(2, 1, dtype=torch.int32), 4, 2, 4)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        Q.linear_act(x, W, activation="relu")
    with pytest.raises(ValueError):
        Q.trellis_words(17, 2)
    assert Q.trellis_words(16, 2) == 17
    from paper_2605_10655_amd.autograd import linear_act8
    with pytest.raises(TypeError):
        linear_act8(x.requires_grad_(), W)


@pytest.mark.parametrize("xs,rs", [((2, 3, 4), (6, 5)), ((6, 4), (2, 3, 5)), ((2, 3, 4), (2, 3, 5)), ((1, 4), (1, 1, 5))])
def test_residual_of_another_shape_gets_its_gradient(xs, rs, monkeypatch):
    """linear_act takes any shapes of as many rows; the residual's gradient has
    the residual's.  (On the host: the product itself is plain here.)"""
    from paper_2605_10655_amd import autograd as A

    def product(x, W, bias, residual, activation, save=False):
        return (x.flatten(0, -2) @ W.t() + residual.flatten(0, -2)).view(*x.shape[:-1], W.shape[0])

    monkeypatch.setattr(A, "linear_act", product)
    monkeypatch.setattr(A, "linear_act_vjp", lambda *a, **kw: (None, None, None))
    x, W = torch.randn(xs), torch.randn(5, 4)
    r = torch.randn(rs, requires_grad=True)
    y = A.linear_act8(x, W, None, r)
    dy = torch.randn(y.shape)
    y.backward(dy)
    assert r.grad.shape == r.shape and torch.equal(r.grad.flatten(), dy.flatten())


def test_a_checkpoint_on_another_device_is_refused_before_the_backward_pass():
    from paper_2605_10655_amd.autograd import linear_act8
    x, W = torch.zeros(4, 8), torch.zeros(6, 8, requires_grad=True)
    a = Q.Act8(torch.zeros(1, 8, 32, dtype=torch.int8, device="meta"), torch.zeros(1, 8, dtype=torch.bfloat16), 4,
               torch.float32)
    with pytest.raises(ValueError, match="device"):
        linear_act8(x, W, x8=a)


def test_anneal_refuses_what_a_layer_loss_cannot_take():
    from paper_2605_10655_amd.qat import QATConfig, anneal_qat
    cfg = QATConfig(state_bits=4, k=2, block=16)
    W, c, X = torch.zeros(4, 32), torch.zeros(16), torch.zeros(5, 32)
    with pytest.raises(ValueError):
        anneal_qat(W, c, cfg, X=X, H=torch.zeros(32, 32))
    with pytest.raises(ValueError):
        anneal_qat(W, c, cfg, activation="silu")
    with pytest.raises(ValueError):
        anneal_qat(W, c, cfg, X=torch.zeros(5, 31))
    with pytest.raises(ValueError):
        anneal_qat(torch.zeros(16, 24), c, cfg, X=torch.zeros(5, 24))


# ---------------------------------------------------------------- the reference
def test_reference_codes():
    x = torch.tensor([[127.0, 127.5, 0.0, 2.0 ** -40], [1.0, 1.0, 0.0, 0.0]])
    codes, scales, v = R.act8_64(x)
    assert scales.tolist() == [[1.0, 2.0, 2.0 ** -126, 2.0 ** -46]]
    assert v[:, 0].tolist() == [127.0, 1.0]
    assert v[0, 1] == 128.0 and codes[0, 1, 0] == 64 and codes[0, 1, 1] == 0     # 0.5 and 63.75 to even, up
    assert v[0, 3] == 2.0 ** -40
    top = torch.tensor([[65504.0], [1.0]], dtype=torch.float16)
    assert R.act8_64(top, fp16=True)[2][0, 0] == 63 * 1024.0
    bad = R.act8_64(torch.tensor([[float("inf")], [3.0]]))
    assert bad[1][0, 0] < 0 and bad[0][0, 0, 0] == -128 and torch.isnan(bad[2][0, 0]) and bad[2][1, 0] == 3.0


@pytest.mark.parametrize("act", R.ACTS)
def test_reference_derivative_matches_differences(act):
    z = torch.linspace(-9, 9, 361, dtype=torch.float64)
    h = 1e-5
    d = (R.act64(z + h, act) - R.act64(z - h, act)) / (2 * h)
    assert (R.slope64(z, act) - d).abs().max() < 1e-9
    assert R.slope64(z, act).abs().max() <= R.LIP


@pytest.mark.parametrize("n,k", [(4, 2), (8, 3), (16, 2), (5, 5), (12, 1)])
def test_reference_strings_are_windows(n, k):
    rng = np.random.default_rng(n * 10 + k)
    s = R.legal_states(rng, 3, 40, n, k)
    w = R.pack64(s, n, k)
    for row, st in zip(w.numpy().view(np.uint32), s):
        text = "".join(format(int(v), "032b") for v in row)
        assert [int(text[t * k:t * k + n], 2) for t in range(40)] == st.tolist()
