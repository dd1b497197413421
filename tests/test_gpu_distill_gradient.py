"""The distillation gradient is the derivative of the loss for every list the calls accept: lists without an entry, lists
whose probabilities add to more than 1, students that have nothing outside the list, and lists with a NaN.  Against
automatic differentiation of the loss in float64, and against differences of the kernel's own loss.

Tolerances, derived before the first run: as for ordinary lists, scaled differences below 2^8 carry an fp32 error of
2^8 * 2^-23 = 3e-5, so losses up to 16 and gradients (by their largest element) are within 1e-4, and a bf16 gradient within
2^-8 of itself as well.
"""
import math

import numpy as np
import pytest
import torch

from _distill_ref import close, distill64

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
ABS = 1e-4
BF16 = 2.0 ** -8


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def logits(rows, vocab, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(rows, vocab, generator=g) * 2
    z.scatter_(1, torch.randint(0, vocab, (rows, 3), generator=g), 9.0)
    return z.to(dtype)


def check(P, z, idx, lp, tau, tail, d_loss):
    loss, grad = distill64(z, idx, lp, tau, tail, d_loss)
    args = (z.to(DEV), idx.to(DEV), lp.to(DEV))
    dd = d_loss.to(DEV)
    kw = dict(temperature=tau, tail=tail)
    size = float(np.nanmax(np.abs(grad), initial=0.0))
    tol_g = ABS * max(1.0, size) + (BF16 if z.dtype == torch.bfloat16 else 0.0) * np.abs(grad)
    tol_l = ABS * np.maximum(1.0, np.abs(loss))
    f = P.camera_distill_forward(*args, **kw)
    close(f["loss"], loss, tol_l, "loss")
    s_loss, s_grad = P.camera_distill_step(*args, dd, **kw)
    close(s_loss, loss, tol_l, "step loss")
    close(s_grad, grad, tol_g, "step")
    b = P.camera_distill_backward(*args, dd, f["lse"], f.get("log_tail"), **kw)
    close(b, grad, tol_g, "backward")
    return s_grad


SHAPES = [(5, 1001), (5, 60000), (700, 301)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab", SHAPES)
@pytest.mark.parametrize("tail", [False, True])
def test_lists_without_an_entry(P, dtype, rows, vocab, tail):
    z = logits(rows, vocab, dtype, 1)
    g = torch.Generator().manual_seed(2)
    k = 9
    idx = torch.stack([torch.randperm(vocab, generator=g)[:k] for _ in range(rows)]).int()
    lp = torch.log_softmax(torch.randn(rows, k, generator=g), 1) - 0.2
    idx[0], lp[0] = -1, -math.inf            # as camera_token_logprobs writes a row that has no distribution
    lp[1] = -math.inf                        # tokens, but none with any probability
    idx[2] = vocab                           # every index outside the vocabulary
    lp[3, 1:] = -math.inf                    # one entry
    got = check(P, z, idx, lp, 1.3, tail, torch.full((rows,), 0.7))
    if not tail:
        assert not got[:3].any()             # a loss that is 0 whatever the logits


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab", SHAPES)
@pytest.mark.parametrize("mass", [1.15, 3.0, 1.0, 0.5])
def test_lists_of_any_mass(P, dtype, rows, vocab, mass):
    z = logits(rows, vocab, dtype, 3)
    g = torch.Generator().manual_seed(4)
    k = 20
    idx = torch.stack([torch.randperm(vocab, generator=g)[:k] for _ in range(rows)]).int()
    lp = torch.log_softmax(torch.randn(rows, k, generator=g), 1) + math.log(mass)
    check(P, z, idx, lp, 0.8, True, torch.rand(rows, generator=g) + 0.5)
    check(P, z, idx, lp, 0.8, False, torch.rand(rows, generator=g) + 0.5)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [40, 60000])
@pytest.mark.parametrize("tail", [False, True])
def test_nothing_outside_the_list(P, dtype, vocab, tail):
    rows, k = 4, 8
    g = torch.Generator().manual_seed(5)
    z = torch.full((rows, vocab), -math.inf)
    idx = torch.stack([torch.randperm(vocab, generator=g)[:k] for _ in range(rows)]).int()
    z.scatter_(1, idx.long(), torch.randn(rows, k, generator=g))
    z[1] = torch.where(z[1] == -math.inf, torch.finfo(dtype).min, z[1])
    lp = torch.log_softmax(torch.randn(rows, k, generator=g), 1) + math.log(0.8)
    check(P, z.to(dtype), idx, lp, 1.0, tail, torch.ones(rows))


@pytest.mark.parametrize("rows,vocab", SHAPES)
@pytest.mark.parametrize("tail", [False, True])
def test_a_nan_in_the_list_reaches_loss_and_gradient(P, rows, vocab, tail):
    """A teacher's row with a NaN comes out of camera_token_logprobs as -1 / NaN; the others are left alone."""
    z = logits(rows, vocab, torch.float32, 6).to(DEV)
    teacher = logits(rows, vocab, torch.float32, 7).to(DEV)
    teacher[1, 5] = math.nan
    top = P.camera_token_logprobs(teacher, top_n=12)
    assert (top["top_idx"][1] == -1).all() and top["top_logprob"][1].isnan().all()
    idx, lp = top["top_idx"], top["top_logprob"].clone()
    lp[2, 3] = math.nan                       # an entry of the vocabulary
    d_loss = torch.ones(rows, device=DEV)
    f = P.camera_distill_forward(z, idx, lp, tail=tail)
    loss, step = P.camera_distill_step(z, idx, lp, d_loss, tail=tail)
    back = P.camera_distill_backward(z, idx, lp, d_loss, f["lse"], f.get("log_tail"), tail=tail)
    bad = torch.zeros(rows, dtype=torch.bool, device=DEV)
    bad[1] = bad[2] = True
    for got in (f["loss"], loss):
        assert torch.equal(got.isnan(), bad)
    for got in (step, back):
        assert got[bad].isnan().all() and not got[~bad].isnan().any()


@pytest.mark.parametrize("tail", [False, True])
def test_gradient_against_differences(P, tail):
    """Central differences of the kernel's own loss: h = 0.05 leaves a truncation error of h^2 / 6 times the third
    derivative (at most the list's mass, 1.5 here): 7e-4, and the loss error 1e-6 / h = 2e-5 at losses of about 1."""
    vocab, k = 40, 6
    g = torch.Generator().manual_seed(8)
    z = torch.randn(1, vocab, generator=g)
    lists = {"no entry": (torch.full((1, k), -1, dtype=torch.int32), torch.full((1, k), -math.inf)),
             "mass 1.5": (torch.arange(k, dtype=torch.int32)[None], torch.full((1, k), math.log(1.5 / k)))}
    masked = z.clone()
    masked[0, k:] = -math.inf
    h = 0.05
    steps = torch.eye(vocab) * h
    for name, (idx, lp), z0 in [(n, l, z) for n, l in lists.items()] + \
            [("nothing outside", (torch.arange(k, dtype=torch.int32)[None], torch.full((1, k), math.log(0.8 / k))), masked)]:
        rep = lambda t: t.to(DEV).expand(vocab, -1).contiguous()
        _, grad = P.camera_distill_step(z0.to(DEV), idx.to(DEV), lp.to(DEV), torch.ones(1, device=DEV), tail=tail)
        up = P.camera_distill_forward((z0 + steps).to(DEV), rep(idx), rep(lp), tail=tail)["loss"]
        down = P.camera_distill_forward((z0 - steps).to(DEV), rep(idx), rep(lp), tail=tail)["loss"]
        close((up - down) / (2 * h), grad[0].double().cpu().numpy(), 9e-4, name)
