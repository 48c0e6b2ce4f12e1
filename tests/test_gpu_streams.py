"""GPU checks of calls on a stream other than the current one: outputs and
workspaces belong to the stream that the call runs on."""
import numpy as np
import pytest

import paper_2605_10655_amd as P
from paper_2605_10655_amd import workloads as WL

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2605_10655_amd.ldlq import block_ldl, ldlq_viterbi  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    P.load_library()
    yield


def _entry_points():
    n, k, B, L, T = 12, 2, 40, 32, 0.1
    w, c, g = (torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in WL.random_case(123, B, L, n))
    r = np.random.default_rng(5)
    cv = torch.from_numpy(r.standard_normal((1 << 8, 2)).astype(np.float32)).cuda()
    X = r.standard_normal((256, 64))
    H = torch.from_numpy((X.T @ X / 256).astype(np.float32)).cuda()
    W = torch.from_numpy(r.standard_normal((16, 64)).astype(np.float32)).cuda()
    hard = P.viterbi_decode(w, c, n, k)[1]
    return {
        "bcjr_soft_codeword": lambda **s: P.bcjr_soft_codeword(w, c, n, k, T, **s),
        "bcjr_soft_codeword_vjp": lambda **s: P.bcjr_soft_codeword_vjp(w, c, n, k, T, g, **s),
        "bcjr_soft_codeword_fwd_vjp": lambda **s: P.bcjr_soft_codeword_fwd_vjp(w, c, n, k, T, g, **s),
        "bcjr_ste_vjp": lambda **s: P.bcjr_ste_vjp(w, c, n, k, T, hard, g, **s),
        "viterbi_decode": lambda **s: P.viterbi_decode(w, c, n, k, **s),
        "bcjr_vec_soft_codeword": lambda **s: P.bcjr_vec_soft_codeword(w, cv, 8, 4, 2, T, **s),
        "bcjr_vec_soft_codeword_vjp": lambda **s: P.bcjr_vec_soft_codeword_vjp(w, cv, 8, 4, 2, T, g, **s),
        "bcjr_vec_viterbi_decode": lambda **s: P.bcjr_vec_viterbi_decode(w, cv, 8, 4, 2, **s),
        "bcjr_gaussian_codebook": lambda **s: P.bcjr_gaussian_codebook(12, 2, **s),
        "block_ldl": lambda **s: block_ldl(H, 16, 0.01, **s),
        "ldlq_viterbi": lambda **s: ldlq_viterbi(W, cv, 8, 4, H, 32, 2, return_targets=True, **s),
    }


def _tensors(out):
    return [t for t in (out if isinstance(out, tuple) else (out,)) if t is not None]


@pytest.mark.parametrize("name", ["bcjr_soft_codeword", "bcjr_soft_codeword_vjp", "bcjr_soft_codeword_fwd_vjp",
                                  "bcjr_ste_vjp", "viterbi_decode", "bcjr_vec_soft_codeword",
                                  "bcjr_vec_soft_codeword_vjp", "bcjr_vec_viterbi_decode",
                                  "bcjr_gaussian_codebook", "block_ldl", "ldlq_viterbi"])
def test_calls_on_a_stream_allocate_from_its_pool(name, monkeypatch):
    """What the current stream has freed, and may still be writing, is not what
    a call on another stream gets for its outputs and its workspace."""
    call = _entry_points()[name]
    print(f"[pool] {name}", flush=True)
    s = torch.cuda.Stream()
    first = _tensors(call())
    want, freed = [t.clone() for t in first], {t.data_ptr() for t in first}
    del first
    torch.cuda.synchronize()
    asked = []
    for maker in ("empty", "empty_like"):
        real = getattr(torch, maker)
        monkeypatch.setattr(torch, maker, lambda *a, real=real, **kw: asked.append(torch.cuda.current_stream()) or real(*a, **kw))
    got = _tensors(call(stream=s))
    monkeypatch.undo()
    s.synchronize()
    assert asked and all(a == s for a in asked)
    assert not freed & {t.data_ptr() for t in got}
    assert torch.cuda.current_stream() != s
    for a, b in zip(got, want):
        if name.endswith("vjp"):   # dCodebook's sums may be added in another order
            assert float((a - b).abs().max()) <= 1e-5 * float(b.abs().max())
        else:
            assert torch.equal(a, b)


def test_given_outputs_and_workspace_are_used():
    """The caller's own memory on another stream."""
    n, k, B, L, T = 12, 2, 40, 32, 0.1
    w, c, _ = (torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in WL.random_case(7, B, L, n))
    want = P.bcjr_soft_codeword(w, c, n, k, T)
    out, ws = torch.empty_like(w), torch.empty(P.bcjr_workspace_bytes(B, L, n, k, P.OP_FWD), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got, logZ = P.bcjr_soft_codeword(w, c, n, k, T, w_soft=out, workspace=ws, stream=s)
    s.synchronize()
    assert got is out and torch.equal(out, want[0]) and torch.equal(logZ, want[1])


def test_a_run_that_ends_early_is_waited_for(monkeypatch):
    """anneal_qat on another stream, ended by an error: the caller's stream is
    ordered behind what was queued, as the inputs may be freed next."""
    from paper_2605_10655_amd import qat
    s, here = torch.cuda.Stream(), torch.cuda.current_stream()
    waits, real = [], torch.cuda.Stream.wait_stream
    monkeypatch.setattr(torch.cuda.Stream, "wait_stream", lambda a, b: waits.append((a, b)) or real(a, b))

    def ends(*a, **kw):
        raise RuntimeError("ended")

    monkeypatch.setattr(qat, "qat_adam_step", ends)
    g = torch.Generator().manual_seed(1)
    W, c = torch.randn(4, 32, generator=g).cuda(), torch.randn(16, generator=g).cuda()
    cfg = qat.QATConfig(state_bits=4, k=2, block=16, steps=2, T0=0.2, T_end=0.1)
    with pytest.raises(RuntimeError, match="ended"):
        qat.anneal_qat(W, c, cfg, stream=s)
    assert waits == [(s, here), (here, s)]
    torch.cuda.synchronize()
