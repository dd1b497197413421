"""Refusals of the recovery operators: bad arguments come back as an error before anything touches a GPU."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def logprobs(P, logits=4096, dtype=1, ld=100, rows=4, vocab=100, targets=4096, top_n=2, tau=1.0, logprob=4096, entropy=4096,
             top_idx=4096, top_logprob=4096):
    return P.lib.camera_token_logprobs(logits, dtype, ld, rows, vocab, targets, top_n, C.c_float(tau), logprob, entropy,
                                       top_idx, top_logprob, None)


def test_token_logprobs_refusals(P):
    assert logprobs(P, rows=0, logits=None) == 0                       # nothing to do
    assert logprobs(P, dtype=2) == -1 and logprobs(P, rows=-1) == -1 and logprobs(P, vocab=0) == -1
    assert logprobs(P, ld=99) == -1                                    # rows overlap
    for tau in (0.0, -1.0, float("nan"), float("inf")):
        assert logprobs(P, tau=tau) == -1
    assert logprobs(P, targets=None) == -1 and logprobs(P, logprob=None) == -1      # both or neither
    assert logprobs(P, top_idx=None) == -1 and logprobs(P, top_logprob=None) == -1
    assert logprobs(P, top_n=-1) == -1 and logprobs(P, top_n=129) == -2
    assert logprobs(P, vocab=(1 << 20) + 1, ld=1 << 21) == -2
    assert logprobs(P, logits=None) == -1 and logprobs(P, logits=4097) == -1        # bf16 at an odd address
    assert logprobs(P, logits=4098, dtype=0) == -1                                  # fp32 at an address not of fp32


def distill(P, **kw):
    from paper_2508_02322_b200.binding import camera_distill_t
    a = dict(logits=4096, ld=100, n_rows=4, dtype=1, vocab=100, teacher_idx=4096, teacher_logprob=4096, k=8, temperature=1.0,
             flags=1)
    a.update(kw)
    return camera_distill_t(*[a[n] for n, _ in camera_distill_t._fields_])


def test_distill_refusals(P):
    lib = P.lib
    fwd = lambda d, loss=4096: lib.camera_distill_forward(C.byref(d), loss, None, None, None)
    assert lib.camera_distill_forward(None, 4096, None, None, None) == -1
    assert fwd(distill(P, n_rows=0, logits=None), None) == 0
    for bad in (dict(k=0), dict(flags=2), dict(temperature=0.0), dict(ld=50), dict(dtype=3), dict(logits=None),
                dict(teacher_idx=None), dict(teacher_logprob=None), dict(n_rows=-2)):
        assert fwd(distill(P, **bad)) == -1, bad
    assert fwd(distill(P, k=129)) == -2 and fwd(distill(P, vocab=1 << 21, ld=1 << 21)) == -2
    assert fwd(distill(P), None) == -1
    bwd = lambda d, dl=4096, lse=4096, tail=4096, g=8192, ld=100: lib.camera_distill_backward(C.byref(d), dl, lse, tail, g, ld, None)
    for bad in (dict(dl=None), dict(lse=None), dict(tail=None), dict(g=None), dict(ld=99), dict(g=8193), dict(g=4096, ld=101)):
        assert bwd(distill(P), **bad) == -1, bad
    step = lambda d, dl=4096, loss=4096, g=8192, ld=100: lib.camera_distill_step(C.byref(d), dl, loss, g, ld, None)
    for bad in (dict(dl=None), dict(loss=None), dict(g=None), dict(ld=99), dict(g=4096, ld=101)):
        assert step(distill(P), **bad) == -1, bad


def test_tensors_are_checked_in_python(P):
    z = torch.zeros(4, 10)
    with pytest.raises(ValueError):
        P.camera_token_logprobs(z)                                     # not on the GPU
    with pytest.raises(ValueError):
        P.camera_distill_forward(z, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2))


def ffn_struct(P, d_model=64, d_ff=40, down_ld=48, w=4096):
    from paper_2508_02322_b200.binding import camera_ffn_t
    return camera_ffn_t(d_model, d_ff, down_ld, w, w, w)


def test_ffn_refusals(P):
    lib = P.lib
    ok = ffn_struct(P)
    size = lib.camera_ffn_workspace_bytes(C.byref(ok), 100, 0)
    both = lib.camera_ffn_workspace_bytes(C.byref(ok), 100, 1)
    assert both > size >= 100 * 40 * 2 and lib.camera_ffn_saved_bytes(C.byref(ok), 100) >= 2 * 100 * 40 * 2
    assert lib.camera_ffn_workspace_bytes(None, 100, 0) == 0
    for bad in (dict(d_model=60), dict(d_ff=0), dict(down_ld=32), dict(down_ld=44), dict(w=None), dict(w=4100), dict(d_ff=41, down_ld=0)):
        assert lib.camera_ffn_workspace_bytes(C.byref(ffn_struct(P, **bad)), 100, 0) == 0, bad
    assert lib.camera_ffn_workspace_bytes(C.byref(ok), -1, 0) == 0

    def fwd(f=ok, x=4096, n=100, y=4096, saved=None, ws=4096, nbytes=size):
        return lib.camera_ffn_forward(C.byref(f), x, n, y, saved, ws, nbytes, None)
    assert fwd(ws=None) == -3 and fwd(nbytes=size - 1) == -3 and fwd(ws=4096 + 64) == -3
    assert fwd(x=None) == -1 and fwd(y=None) == -1 and fwd(x=4104) == -1 and fwd(saved=4112) == -1
    assert fwd(ffn_struct(P, d_model=60)) == -2 and fwd(ffn_struct(P, w=None)) == -1

    def bwd(x=4096, dy=4096, n=100, saved=4096, dx=4096, dg=4096, du=4096, dd=4096, ws=4096, nbytes=both):
        return lib.camera_ffn_backward(C.byref(ok), x, dy, n, saved, dx, dg, du, dd, ws, nbytes, None)
    assert bwd(nbytes=size) == -3 and bwd(dg=None) == -1 and bwd(dd=None) == -1 and bwd(dd=4104) == -1
    assert bwd(dx=None, dg=None, du=None, dd=None) == -1          # nothing asked for
    assert bwd(saved=None) == -1 and bwd(dy=None) == -1 and bwd(dx=4104) == -1


def test_ffn_tensors_are_checked_in_python(P):
    w = torch.zeros(16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        P.Ffn(w, w, torch.zeros(64, 8, dtype=torch.bfloat16))           # fewer columns than micro-experts
    with pytest.raises(ValueError):
        P.Ffn(w.float(), w, torch.zeros(64, 16, dtype=torch.bfloat16))
    ffn = P.Ffn(w, w, torch.zeros(64, 16, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        P.camera_ffn_forward(ffn, torch.zeros(4, 32, dtype=torch.bfloat16))
    with pytest.raises(P.CameraError):
        P.camera_ffn_workspace_bytes(P.Ffn(torch.zeros(16, 60, dtype=torch.bfloat16), torch.zeros(16, 60, dtype=torch.bfloat16),
                                           torch.zeros(60, 16, dtype=torch.bfloat16)), 8)
