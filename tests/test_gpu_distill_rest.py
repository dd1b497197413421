"""The rest class where the student's share outside the teacher's list is tiny: loss and gradient down to shares of e^-700,
nothing below 2^-1022.

Tolerances, derived before the first run.  Tokens outside lie within a few nats of each other, the list far above them.
A token's weight among those outside is 2^(x c - k) with x c and k of up to 2^10 in size: an fp32 error of 2^10 * 2^-23 =
1.2e-4 where neither is formed from differences, which is the relative error of the gradient outside the list; bound 3e-4
of each element (the logarithm of the share enters the loss with the same relative error or less), plus 2^-8 in bf16.
On the list gradients are differences of probabilities: 1e-4 absolute.  camera_distill_backward takes lse and log_tail in
fp32: their rounding, 2^-24 of up to 2^10 nats, adds 6e-5.
"""
import math

import numpy as np
import pytest
import torch

from _distill_ref import close, distill64

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
REL = 3e-4
BF16 = 2.0 ** -8


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def make(rows, vocab, k, gap, centre, seed, dtype):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(rows, vocab, generator=g) + centre - gap
    idx = torch.stack([torch.randperm(vocab, generator=g)[:k] for _ in range(rows)])
    idx[0] = torch.arange(k)                       # the row's first vectors ...
    idx[1] = torch.arange(vocab - k, vocab)        # ... and its last
    z.scatter_(1, idx, centre + torch.randn(rows, k, generator=g))
    lp = torch.log_softmax(torch.randn(rows, k, generator=g), 1) + math.log(0.9)
    return z.to(dtype), idx.int(), lp


@pytest.mark.parametrize("dtype,pad,shift", [(torch.float32, 0, 0), (torch.float32, 1, 3), (torch.bfloat16, 3, 1)])
@pytest.mark.parametrize("rows,vocab,k", [(3, 523, 16), (3, 151936, 64), (400, 1300, 7)])
@pytest.mark.parametrize("gap", [20.0, 75.0, 85.0, 90.0, 100.0, 200.0, 700.0])
@pytest.mark.parametrize("centre", [0.0, 60.0])
def test_small_shares(P, dtype, pad, shift, rows, vocab, k, gap, centre):
    z, idx, lp = make(rows, vocab, k, gap, centre, int(gap) + vocab, dtype)
    d_loss = torch.ones(rows)
    some = min(rows, 6)
    loss, grad = distill64(z[:some], idx[:some], lp[:some], 1.0, True, d_loss)
    buf = torch.zeros(rows * (vocab + pad) + shift, dtype=dtype, device=DEV)
    view = buf[shift:].view(rows, vocab + pad)[:, :vocab]
    view.copy_(z)
    args = (view, idx.to(DEV), lp.to(DEV))
    listed = np.zeros((some, vocab), dtype=bool)
    for r in range(some):
        listed[r, idx[r].numpy()] = True
    rel = REL + (BF16 if dtype == torch.bfloat16 else 0.0)
    # a gradient outside the list is R - rest times a weight: R's own error counts where the two are of one size
    tol = np.where(listed, 1e-4, 0.0) + rel * np.abs(grad) + 1e-12
    f = P.camera_distill_forward(*args, tail=True)
    close(f["loss"][:some], loss, REL * np.maximum(1.0, np.abs(loss)), "loss")
    s_loss, s_grad = P.camera_distill_step(*args, d_loss.to(DEV), tail=True)
    assert torch.equal(s_loss, f["loss"])
    close(s_grad[:some], grad, tol, "step")
    back = P.camera_distill_backward(*args, d_loss.to(DEV), f["lse"], f["log_tail"], tail=True)
    close(back[:some], grad, tol, "backward")
    # the share's logarithm itself, as backward takes it
    zd = z[:some].double()
    want = torch.logsumexp(zd.masked_fill(torch.from_numpy(listed), -math.inf), 1).numpy()
    close(f["log_tail"][:some], want, 1e-4 + 2.0 ** -22 * np.abs(want), "log_tail")
    # and with the exact logarithms from elsewhere
    exact = (torch.logsumexp(zd, 1).float().to(DEV), torch.from_numpy(want).float().to(DEV))
    if some == rows:
        back = P.camera_distill_backward(*args, d_loss.to(DEV), *exact, tail=True)
        close(back, grad, tol, "backward from given logarithms")


@pytest.mark.parametrize("gap", [750.0, 5000.0, 1e30])
@pytest.mark.parametrize("vocab", [523, 60000])
def test_no_share_left(P, gap, vocab):
    """Below 2^-1022 the student has nothing outside: the rest's term is dropped, as for logits of minus infinity."""
    z, idx, lp = make(3, vocab, 16, gap, 0.0, 1, torch.float32)
    d_loss = torch.ones(3)
    loss, grad = distill64(z, idx, lp, 1.0, True, d_loss)
    args = (z.to(DEV), idx.to(DEV), lp.to(DEV))
    f = P.camera_distill_forward(*args, tail=True)
    s_loss, s_grad = P.camera_distill_step(*args, d_loss.to(DEV), tail=True)
    back = P.camera_distill_backward(*args, d_loss.to(DEV), f["lse"], f["log_tail"], tail=True)
    close(f["loss"], loss, 1e-4 * np.maximum(1.0, np.abs(loss)))
    assert torch.equal(s_loss, f["loss"])
    for got in (s_grad, back):
        close(got, grad, 1e-4)
        assert torch.equal((got != 0).sum(1), torch.full((3,), 16, device=DEV))
