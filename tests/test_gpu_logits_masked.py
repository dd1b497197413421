"""Rows of logits of which few tokens are allowed: most of a thread's share, and often all of its beginning, is masked.
Log-probabilities with and without entropy and alternatives, distillation in every mode, against float64.

Tolerances, derived before the first run.  Scaled differences to a thread's reference are at most 2^8 in size here and
carry an fp32 error of at most 2^8 * 2^-23 = 3e-5, which is the relative error of a weight; sums, logarithms and
ex2.approx add a few times 2^-22.  Log-probabilities, entropies and losses of size up to 16 are within 1e-4 of the truth, a
gradient within 1e-4 of the largest weight plus its rounding to the output's type (2^-8 relative covers bf16).
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


def masked_logits(vocab, dtype, mask, seed):
    """Rows with about 1 % (the last: 30 %) of the tokens allowed, anywhere, at the row's end or at its start: the bulk of
    them at -5, a few at up to 6.  Others hold `mask`."""
    g = torch.Generator().manual_seed(seed)
    rows = 6
    z = torch.full((rows, vocab), mask)
    n = max(8, vocab // 100)
    allowed = [torch.randperm(vocab, generator=g)[:n], torch.arange(vocab - n, vocab), torch.arange(n),
               torch.randperm(vocab, generator=g)[:n], torch.randperm(vocab, generator=g)[: n // 2 + 4],
               torch.randperm(vocab, generator=g)[: vocab * 3 // 10]]
    top = [2.0, 2.0, 2.0, 6.0, 3.0, 2.5]
    for r in range(rows):
        i = allowed[r]
        z[r, i] = -5.0 + 0.5 * torch.randn(len(i), generator=g)
        z[r, i[torch.randint(0, len(i), (4,), generator=g)]] = top[r]
    z = z.to(dtype)
    targets = torch.stack([i[3] for i in allowed])
    return z, targets


MASKS = [-math.inf, "lowest", -1e4, -80.0]


def mask_value(mask, dtype):
    return torch.finfo(dtype).min if mask == "lowest" else mask


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [32000, 50257, 151936])
@pytest.mark.parametrize("mask", MASKS)
def test_logprobs(P, dtype, vocab, mask):
    z, targets = masked_logits(vocab, dtype, mask_value(mask, dtype), vocab)
    zd, td = z.to(DEV), targets.to(DEV)
    lp = torch.log_softmax(z.double(), 1)
    want = lp.gather(1, targets[:, None]).squeeze(1).numpy()
    ent = -torch.xlogy(lp.exp(), lp.exp()).sum(1).numpy()
    for top_n in (0, 3):
        plain = P.camera_token_logprobs(zd, td, entropy=False, top_n=top_n)
        close(plain["logprob"], want, ABS, "without entropy")
        full = P.camera_token_logprobs(zd, td, top_n=top_n)
        close(full["logprob"], want, ABS, "with entropy")
        close(full["entropy"], ent, ABS, "entropy")
        if top_n:
            idx = torch.sort(z.double(), dim=1, descending=True, stable=True).indices[:, :top_n]
            assert torch.equal(plain["top_idx"].cpu().long(), idx) and torch.equal(full["top_idx"].cpu().long(), idx)
            close(plain["top_logprob"], lp.gather(1, idx).numpy(), ABS, "alternatives")
    # many rows: every CTA walks rows of its own
    many = zd.repeat(100, 1)
    got = P.camera_token_logprobs(many, td.repeat(100), entropy=False)["logprob"]
    close(got, np.tile(want, 100), ABS, "many rows")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [50257, 151936])
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("tail", [False, True])
def test_distillation(P, dtype, vocab, mask, tail):
    z, _ = masked_logits(vocab, dtype, mask_value(mask, dtype), vocab + 1)
    rows, k = z.shape[0], 24
    g = torch.Generator().manual_seed(3)
    # the list: allowed tokens, the largest and others
    idx = torch.empty(rows, k, dtype=torch.int32)
    for r in range(rows):
        allowed = torch.nonzero(z[r].float() > -20).squeeze(1)
        best = z[r].double().topk(2).indices
        other = allowed[torch.randperm(len(allowed), generator=g)]
        other = other[(other != best[0]) & (other != best[1])]
        idx[r] = torch.cat([best, other])[:k].int() if len(allowed) >= k else -1
        idx[r, : min(k, len(allowed))] = torch.cat([best, other])[: min(k, len(allowed))].int()
    lp = torch.log_softmax(torch.randn(rows, k, generator=g), 1) - 0.3
    d_loss = torch.rand(rows, generator=g) + 0.5
    loss, grad = distill64(z, idx, lp, 1.0, tail, d_loss)
    args = (z.to(DEV), idx.to(DEV), lp.to(DEV))
    dd = d_loss.to(DEV)
    tol_g = ABS * max(1.0, float(np.abs(grad).max())) + (BF16 if dtype == torch.bfloat16 else 0.0) * np.abs(grad)
    tol_l = ABS * np.maximum(1.0, np.abs(loss))
    f = P.camera_distill_forward(*args, tail=tail)
    close(f["loss"], loss, tol_l, "loss")
    close(f["lse"], torch.logsumexp(z.double(), 1).numpy(), ABS, "lse")
    s_loss, s_grad = P.camera_distill_step(*args, dd, tail=tail)
    close(s_loss, loss, tol_l, "step")
    close(s_grad, grad, tol_g, "step")
    b = P.camera_distill_backward(*args, dd, f["lse"], f.get("log_tail"), tail=tail)
    close(b, grad, tol_g, "backward")
