"""Distillation from a teacher's list in 64 bits: the loss from its definition, the gradient from automatic
differentiation of that loss."""
import math

import numpy as np
import torch

NONE_LN = -1022 * math.log(2)      # a share below 2^-1022 counts as none


def teacher(idx, lp, vocab, tail):
    """The entries that count (their indices and a mask over the list), p, ln p and the rest of one row in float64."""
    on = (idx >= 0) & (idx < vocab)
    lp = torch.where(on | lp.isnan(), lp.double(), torch.tensor(-math.inf, dtype=torch.float64))
    if tail:
        p = lp.exp()
        return on, p, lp, (1 - p.sum()).clamp_min(0.0)
    zero = torch.zeros((), dtype=torch.float64)
    if (lp == -math.inf).all():
        return on, torch.zeros_like(lp), lp, zero
    lp = torch.log_softmax(lp, 0)
    return on, lp.exp(), lp, zero


def distill_row(z, idx, lp, tau, tail, d_loss):
    """Loss and gradient of one row (z, idx, lp 1-d)."""
    vocab = z.numel()
    z = z.double().detach().clone()
    if z.isnan().any() or (z == math.inf).any() or lp.isnan().any():
        return math.nan, torch.full((vocab,), math.nan, dtype=torch.float64)
    if (z == -math.inf).all():
        return 0.0, torch.zeros(vocab, dtype=torch.float64)
    z.requires_grad_(True)
    on, p, ln_p, rest = teacher(idx, lp, vocab, tail)
    lq = torch.log_softmax(z / tau, 0)
    use = on & (p > 0)
    loss = (p[use] * (ln_p[use] - lq[idx[use].long()])).sum() + 0.0 * lq[z > -math.inf].sum()
    outside = torch.ones(vocab, dtype=torch.bool)
    outside[idx[on].long()] = False
    outside &= z > -math.inf
    if rest > 0 and outside.any():
        ln_R = torch.logsumexp(lq[outside], 0)
        if ln_R >= NONE_LN:
            loss = loss + rest * (rest.log() - ln_R)
    grad = torch.autograd.grad(loss, z)[0]
    return loss.item(), grad * d_loss


def distill64(z, idx, lp, tau, tail, d_loss):
    """Loss [rows] and gradient [rows, vocab] as float64 numpy arrays."""
    rows = [distill_row(z[r], idx[r], lp[r], tau, tail, float(d_loss[r])) for r in range(z.shape[0])]
    return np.array([l for l, _ in rows]), torch.stack([g for _, g in rows]).numpy()


def close(got, want, tol, what=""):
    got, want = got.double().cpu().numpy(), np.asarray(want)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        near = np.abs(got - want) <= tol
    ok = same | near
    assert ok.all(), (what, int((~ok).sum()), got[~ok][:5], want[~ok][:5], np.argwhere(~ok)[:5].tolist())
