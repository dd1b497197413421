"""Log-probabilities of tokens that lie very far below the row's largest logit, against float64.

Tolerance, derived before the first run: two fp32 products and a difference, 2^-22 of the value."""
import numpy as np
import pytest
import torch

from _distill_ref import close

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def in_fp32(t):
    """Rounded as the outputs are: what lies beyond fp32's largest value is infinite, what rounds to it is not."""
    return t.float().double().numpy()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [11, 600, 40000])
@pytest.mark.parametrize("tau", [1.0, 0.5, 3.0])
def test_far_below_the_largest(P, dtype, vocab, tau):
    low = torch.finfo(dtype).min
    largest = [2.0 ** 106, 2.0 ** 101, 1e31, 5.0, -2.0 ** 105]
    z = torch.zeros(len(largest), vocab)
    for r, top in enumerate(largest):
        z[r] = min(0.0, 2 * top)
        z[r, 3] = top
        z[r, 4] = -abs(top) * 2
        z[r, 5] = low
    z = z.to(dtype)
    d = z.double() / tau
    lp = torch.log_softmax(d, 1)
    for t in (3, 0, 4, 5):
        targets = torch.full((len(largest),), t)
        got = P.camera_token_logprobs(z.to(DEV), targets.to(DEV), temperature=tau, top_n=vocab if vocab < 128 else 0)
        want = in_fp32(lp[:, t])
        close(got["logprob"], want, 2.0 ** -22 * np.abs(np.where(np.isinf(want), 0.0, want)) + 1e-5, t)
        if vocab < 128:
            idx = got["top_idx"].cpu().long()
            all_ = in_fp32(lp.gather(1, idx))
            close(got["top_logprob"], all_, 2.0 ** -22 * np.abs(np.where(np.isinf(all_), 0.0, all_)) + 1e-5, "alternatives")
