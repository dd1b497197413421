"""Token log-probabilities and top-k distillation against plain float64 restatements on the CPU.

Tolerances, derived before the first run.  Logits here are at most 60 in size, so that a scaled difference (x - m) c is
below 2^8 and carries an fp32 error of at most 2^8 * 2^-23 = 3e-5 (three roundings of half an ulp), which is also the
relative error of a weight 2^d; the sums add a few times 2^-23 per level and ex2.approx 2^-22.  A log-probability, an
entropy or a loss of size up to 2^7 therefore is within 1e-4 of the truth; differences that matter are far larger.  A
gradient is q - p scaled: its absolute error is at most 1e-4 of the largest weight, plus the rounding to the output's
type (2^-9 relative in bf16).  Indices and what is masked have to be exact.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
ABS = 1e-4
BF16 = 2.0 ** -8           # half an ulp is 2^-9 relative; twice that for values next to a power of two


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def padded(z, pad, dtype, shift=0):
    """z as a view whose rows are `pad` elements longer and whose first element lies `shift` elements into its buffer."""
    rows, n = z.shape
    buf = torch.full((rows * (n + pad) + shift,), 3.0, dtype=dtype, device=DEV)
    view = buf[shift:].view(rows, n + pad)[:, :n]
    view.copy_(z)
    return view


def random_logits(rows, vocab, seed, dtype, peaks=4):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(rows, vocab, generator=g) * 2
    for _ in range(peaks):
        i = torch.randint(0, vocab, (rows, 1), generator=g)
        z.scatter_(1, i, torch.rand(rows, 1, generator=g) * 20)
    return z.to(dtype)


# ------------------------------------------------------------------------------------------------ plain forms
def ref_logprobs(z, targets, n, tau):
    z = z.double().numpy()
    rows, vocab = z.shape
    lp_out, ent = np.zeros(rows), np.zeros(rows)
    idx = np.full((rows, n), -1, dtype=np.int32)
    val = np.full((rows, n), -np.inf)
    for r in range(rows):
        x = z[r] / tau
        if np.isnan(x).any() or (x == np.inf).any():
            lp_out[r] = np.nan if 0 <= targets[r] < vocab else 0.0
            ent[r] = np.nan
            val[r] = np.nan
            continue
        if (x == -np.inf).all():
            lp_out[r] = -np.inf if 0 <= targets[r] < vocab else 0.0
            continue
        m = x.max()
        lp = (x - m) - math.log(np.exp(x - m).sum())        # m may be so large that m + log(sum) is m
        p = np.exp(lp)
        ent[r] = -(p[p > 0] * lp[p > 0]).sum()
        if 0 <= targets[r] < vocab:
            lp_out[r] = lp[targets[r]]
        order = np.lexsort((np.arange(vocab), -z[r]))[:n]
        order = order[z[r][order] > -np.inf]
        idx[r, :len(order)] = order
        val[r, :len(order)] = lp[order]
    return lp_out, ent, idx, val


def close(got, want, tol):
    got, want = got.double().cpu().numpy(), np.asarray(want)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        near = np.abs(got - want) <= tol
    assert (same | near).all(), (got[~(same | near)][:5], want[~(same | near)][:5])


def check_logprobs(P, view, targets, n, tau):
    out = P.camera_token_logprobs(view, targets.to(DEV), top_n=n, temperature=tau)
    lp, ent, idx, val = ref_logprobs(view.float().cpu(), targets.numpy(), n, tau)
    close(out["logprob"], lp, ABS)
    close(out["entropy"], ent, ABS)
    if n:
        assert np.array_equal(out["top_idx"].cpu().numpy(), idx)
        close(out["top_logprob"], val, ABS)
    else:
        assert "top_idx" not in out
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab,n,tau,pad,shift", [
    (1, 1, 1, 1.0, 0, 0), (3, 2, 5, 0.5, 0, 1), (5, 7, 7, 1.0, 1, 0), (1, 8, 3, 1.0, 0, 0), (2, 9, 0, 1.7, 0, 3),
    (4, 1000, 20, 1.0, 0, 0), (3, 4095, 64, 2.0, 1, 5), (2, 4096, 128, 1.0, 8, 0), (7, 16385, 33, 0.7, 3, 1),
    (1, 151936, 8, 1.0, 0, 0), (2, 152064, 128, 1.0, 0, 0), (300, 523, 4, 1.0, 0, 0), (1, 1 << 20, 10, 1.0, 0, 0)])
def test_logprobs_sizes_strides_alignments(P, dtype, rows, vocab, n, tau, pad, shift):
    z = random_logits(rows, vocab, rows * 131 + vocab, dtype)
    g = torch.Generator().manual_seed(5)
    targets = torch.randint(0, vocab, (rows,), generator=g)
    check_logprobs(P, padded(z, pad, dtype, shift), targets, n, tau)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [600, 20001])
def test_logprobs_masks_infinities_and_ties(P, dtype, vocab):
    low = torch.finfo(dtype).min
    z = random_logits(14, vocab, 3, dtype)
    z[0] = -math.inf                                    # nothing left
    z[1] = low                                          # a mask of the lowest value everywhere: uniform
    z[2, 5:] = -math.inf                                # five tokens left, fewer than the alternatives asked for
    z[3, 1:] = low                                      # one token and lowest values: those can be listed
    z[4] = 0.0                                          # every logit equal: ties by index
    z[5] = -0.0
    z[5, ::3] = 0.0                                     # both zeros are one value
    z[6, 17] = math.nan
    z[7, 18] = math.inf
    z[8] = torch.arange(vocab).float().remainder(3).to(dtype)     # long runs of ties at the top
    z[9, : vocab // 2] = -math.inf
    z[10] = -math.inf
    z[10, vocab - 1] = 2.0                              # a single token, the last
    z[11] = torch.finfo(dtype).max
    z[12] = 50.0
    z[12, 0] = -50.0
    targets = torch.zeros(14, dtype=torch.long)
    targets[2], targets[9], targets[10], targets[13] = 3, vocab - 2, vocab - 1, -100
    view = padded(z, 1, dtype)
    for n in (1, 20, 128):
        if n == 20:
            check_logprobs(P, view[[0, 1, 2, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13]].contiguous(),
                           targets[[0, 1, 2, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13]], n, 1.0)
        check_logprobs(P, view, targets, n, 1.0)
    # at a low temperature the lowest values overflow once scaled: still no NaN, and a uniform row stays uniform
    out = P.camera_token_logprobs(view[1:2], targets[1:2].to(DEV), top_n=2, temperature=0.25)
    close(out["entropy"], [math.log(vocab)], ABS)
    close(out["logprob"], [-math.log(vocab)], ABS)
    targets[0] = vocab                                   # outside: ignored
    out = P.camera_token_logprobs(view[:1], targets[:1].to(DEV), top_n=1)
    assert out["logprob"].item() == 0.0 and out["entropy"].item() == 0.0 and out["top_idx"].item() == -1
    assert out["top_logprob"].item() == -math.inf


def test_logprobs_optional_outputs_empty_batches_and_streams(P):
    z = random_logits(6, 777, 1, torch.bfloat16).to(DEV)
    assert set(P.camera_token_logprobs(z)) == {"entropy"}
    assert P.camera_token_logprobs(z, entropy=False, top_n=3)["top_idx"].shape == (6, 3)
    out = P.camera_token_logprobs(z[:0], torch.empty(0, dtype=torch.long, device=DEV), top_n=2)
    assert out["logprob"].shape == (0,) and out["top_idx"].shape == (0, 2)
    ref = P.camera_token_logprobs(z, top_n=9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = P.camera_token_logprobs(z, top_n=9, stream=side)
    side.synchronize()
    assert all(torch.equal(ref[k], got[k]) for k in ref)


# ------------------------------------------------------------------------------------------------ distillation
def ref_distill(z, idx, lp, tau, tail, d_loss):
    """Loss and gradient of every row in float64, from the definitions, by hand."""
    z, lp = z.double().numpy(), lp.double().numpy()
    rows, vocab = z.shape
    loss, grad = np.zeros(rows), np.zeros((rows, vocab))
    for r in range(rows):
        x = z[r] / tau
        on = np.array([0 <= i < vocab for i in idx[r].tolist()])
        i, l = idx[r].numpy()[on], lp[r][on]
        if (x * 1.4426950408889634 < -3.4028235e38).all():       # the documented rule for rows without a distribution
            continue
        if tail:
            p, rest = np.exp(l), max(0.0, 1.0 - np.exp(l).sum())
        else:
            rest = 0.0
            if len(l) and np.exp(l).sum() > 0:
                l = l - l.max()
                l = l - math.log(np.exp(l).sum())
            p = np.exp(l)
        m = x.max()
        q = np.exp(x - m) / np.exp(x - m).sum()
        outside = np.ones(vocab, dtype=bool)
        outside[i] = False
        R = q[outside].sum()
        with np.errstate(divide="ignore"):
            loss[r] = sum(pj * (lj - math.log(qj)) if qj > 0 else math.inf for pj, lj, qj in zip(p, l, q[i]) if pj > 0)
        scale = np.ones(vocab)
        if rest > 0 and R > 0:
            loss[r] += rest * math.log(rest / R)
            scale[outside] = 1 - rest / R
        elif rest > 0:
            scale[outside] = 0.0
        g = q * scale
        g[i] = q[i] - p
        grad[r] = g * d_loss[r].item() / tau
    return loss, grad


def make_list(z, k, tau, seed):
    """A teacher's list for a student z: the top of a perturbed copy, with its log-probabilities."""
    g = torch.Generator().manual_seed(seed)
    t = (z.float() + torch.randn(z.shape, generator=g)) / tau
    lp = torch.log_softmax(t.double(), 1)
    top = lp.topk(min(k, z.shape[1]), 1)
    idx = torch.full((z.shape[0], k), -1, dtype=torch.int32)
    out = torch.full((z.shape[0], k), -math.inf)
    idx[:, :top.indices.shape[1]] = top.indices.int()
    out[:, :top.values.shape[1]] = top.values.float()
    return idx, out


def check_distill(P, view, idx, lp, tau, tail, d_loss, tol=ABS):
    z = view.float().cpu()
    loss, grad = ref_distill(z, idx, lp, tau, tail, d_loss)
    di, dl, dd = idx.to(DEV), lp.to(DEV), d_loss.to(DEV)
    kw = dict(temperature=tau, tail=tail)
    live = d_loss.numpy() != 0
    out_tol = tol * max(1.0, float(np.abs(grad).max())) + (BF16 if view.dtype == torch.bfloat16 else 0.0) * np.abs(grad)
    f = P.camera_distill_forward(view, di, dl, **kw)
    close(f["loss"], loss, tol * np.maximum(1.0, np.abs(loss)))
    s_loss, s_grad = P.camera_distill_step(view, di, dl, dd, **kw)
    assert torch.equal(s_loss, torch.where(dd == 0, torch.zeros_like(f["loss"]), f["loss"]))
    close(s_grad, np.where(live[:, None], grad, 0.0), out_tol)
    b_grad = P.camera_distill_backward(view, di, dl, dd, f["lse"], f.get("log_tail"), **kw)
    close(b_grad, np.where(live[:, None], grad, 0.0), out_tol)
    # in place: the gradient takes the logits' room
    again = padded(view, 0, view.dtype)
    _, g = P.camera_distill_step(again, di, dl, dd, d_logits=again, **kw)
    assert g is again
    close(g, s_grad.double().cpu().numpy(), 0.0 if view.stride(0) == again.stride(0) else out_tol)
    return f, s_grad


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("rows,vocab,k,tau,pad,shift", [
    (1, 1, 1, 1.0, 0, 0), (2, 3, 2, 1.0, 0, 1), (3, 9, 9, 2.0, 1, 0), (5, 64, 8, 1.0, 0, 0), (3, 1000, 33, 0.6, 3, 5),
    (2, 4097, 64, 1.0, 0, 0), (2, 20003, 128, 2.5, 5, 1), (1, 151936, 64, 2.0, 0, 0), (260, 130, 4, 1.0, 0, 0)])
def test_distill_sizes_strides_alignments(P, dtype, tail, rows, vocab, k, tau, pad, shift):
    z = random_logits(rows, vocab, vocab + k, dtype)
    idx, lp = make_list(z, k, tau, 9)
    g = torch.Generator().manual_seed(2)
    d_loss = torch.rand(rows, generator=g) + 0.5
    if rows > 2:
        d_loss[1] = 0.0
    if k == vocab and tail:
        lp = lp - 1e-6          # the whole vocabulary is on the list: what rounding leaves over is dropped
    check_distill(P, padded(z, pad, dtype, shift), idx, lp, tau, tail, d_loss)


@pytest.mark.parametrize("dtype,vocab,pad", [(torch.bfloat16, 110001, 7), (torch.float32, 60001, 0)])
def test_more_long_rows_than_run_at_one_time(P, dtype, vocab, pad):
    """Every CTA walks several rows, long ones in pairs of CTAs; some do not count, one holds the lowest value only."""
    rows, k, tau = 321, 40, 1.4
    z = random_logits(rows, vocab, 12, dtype)
    z[200] = torch.finfo(dtype).min
    z[300, vocab // 3:] = -math.inf
    g = torch.Generator().manual_seed(3)
    idx = torch.stack([torch.randperm(vocab // 3, generator=g)[:k] for _ in range(rows)]).int()
    lp = torch.log_softmax(torch.randn(rows, k, generator=g) * 2, 1) - 0.05
    d_loss = torch.rand(rows, generator=g) + 0.5
    d_loss[torch.rand(rows, generator=g) < 0.1] = 0.0
    d_loss[200] = 0.0
    view = padded(z, pad, dtype)
    check_distill(P, view, idx, lp, tau, True, d_loss)
    targets = torch.randint(0, vocab // 3, (rows,), generator=g)
    check_logprobs(P, view, targets, 30, tau)


@pytest.mark.parametrize("offset", [3e3, 1e5, -1e5, 1e8])
@pytest.mark.parametrize("tail", [False, True])
def test_step_does_not_depend_on_where_the_logits_lie(P, tail, offset):
    """Differences decide: logits around a large value have the gradient of the stored values' differences."""
    z = random_logits(5, 5003, 21, torch.float32) + offset
    idx, lp = make_list(z - offset, 30, 1.0, 2)
    d_loss = torch.ones(5)
    loss, grad = ref_distill(z, idx, lp, 1.0, tail, d_loss)
    got, g = P.camera_distill_step(z.to(DEV), idx.to(DEV), lp.to(DEV), d_loss.to(DEV), tail=tail)
    close(got, loss, ABS * np.maximum(1.0, np.abs(loss)))
    close(g, grad, ABS)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tail", [False, True])
def test_distill_masks_and_absent_entries(P, dtype, tail):
    vocab, k = 3001, 16
    low = torch.finfo(dtype).min
    z = random_logits(9, vocab, 4, dtype)
    idx, lp = make_list(z, k, 1.0, 5)
    z[0] = -math.inf                                    # no distribution: no loss, no gradient
    idx[1], lp[1] = -1, -math.inf                       # nothing on the teacher's list
    idx[2, 3:] = -1                                     # a short list
    idx[3, 2] = vocab                                   # outside the vocabulary: no entry
    lp[4, 1] = -math.inf                                # an entry without probability
    z[5, vocab // 2:] = -math.inf                       # masked by minus infinity ...
    idx[5] = torch.arange(k, dtype=torch.int32)
    z[6, vocab // 2:] = low                             # ... and by the lowest value
    idx[6] = torch.arange(k, dtype=torch.int32)
    z[7, k:] = -math.inf                                # the student has nothing outside the list
    idx[7] = torch.arange(k, dtype=torch.int32)
    d_loss = torch.ones(9)
    d_loss[8] = 0.0
    check_distill(P, padded(z, 3, dtype), idx, lp, 1.0, tail, d_loss)
    # rows that do not count may hold anything
    z[8, 5] = math.nan
    view = padded(z, 0, dtype)
    loss, grad = P.camera_distill_step(view, idx.to(DEV), lp.to(DEV), d_loss.to(DEV), tail=tail)
    assert loss[8].item() == 0.0 and (grad[8] == 0).all()
    # rows that count pass a NaN on, and it stays in its row
    d_loss[8] = 1.0
    loss, grad = P.camera_distill_step(view, idx.to(DEV), lp.to(DEV), d_loss.to(DEV), tail=tail)
    assert math.isnan(loss[8].item()) and torch.isnan(grad[8]).any() and not torch.isnan(grad[:8]).any()


@pytest.mark.parametrize("tail", [False, True])
def test_distill_gradient_against_differences(P, tail):
    """Central differences of the kernel's own loss: h = 0.05 leaves a truncation error of h^2 / 6 times the third
    derivative (at most 1 here): 5e-4, and the loss error 1e-6 / h = 2e-5 at losses of about 1."""
    vocab, k, tau = 40, 6, 1.3
    z = random_logits(1, vocab, 8, torch.float32, peaks=2) * 0.5
    idx, lp = make_list(z, k, tau, 1)
    di, dl = idx.to(DEV), lp.to(DEV)
    _, grad = P.camera_distill_step(z.to(DEV), di, dl, torch.ones(1, device=DEV), temperature=tau, tail=tail)
    h = 0.05
    steps = torch.eye(vocab) * h
    rep = lambda t: t.to(DEV).expand(vocab, -1).contiguous()
    up = P.camera_distill_forward((z + steps).to(DEV), rep(idx), rep(lp), temperature=tau, tail=tail)["loss"]
    down = P.camera_distill_forward((z - steps).to(DEV), rep(idx), rep(lp), temperature=tau, tail=tail)["loss"]
    close((up - down) / (2 * h), grad[0].double().cpu().numpy(), 6e-4)


def test_distill_of_the_teacher_itself(P):
    """The lists camera_token_logprobs writes are the ones the loss reads: with the rest as a class a model has no
    divergence from itself; against its renormalised list it has -ln Q, Q the list's probability."""
    z = random_logits(20, 5001, 6, torch.float32).to(DEV)
    top = P.camera_token_logprobs(z, top_n=50, temperature=1.5)
    args = (z, top["top_idx"], top["top_logprob"], torch.ones(20, device=DEV))
    loss, grad = P.camera_distill_step(*args, temperature=1.5, tail=True)
    assert loss.abs().max().item() <= ABS and grad.abs().max().item() <= ABS
    loss, _ = P.camera_distill_step(*args, temperature=1.5, tail=False)
    close(loss, -torch.logsumexp(top["top_logprob"].double(), 1).cpu().numpy(), ABS)
    f = P.camera_distill_forward(z[:0], top["top_idx"][:0], top["top_logprob"][:0], tail=True)
    assert f["loss"].shape == (0,)
