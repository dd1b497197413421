"""Outputs with more than 2^31 elements: offsets of rows do not fit 32 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def test_alternatives_of_more_rows_than_32_bits_address(P):
    rows, n = (1 << 24) + 5, 128                     # rows * n = 2^31 + 640; 17 GB of results
    g = torch.Generator(device=DEV).manual_seed(1)
    z = torch.randint(-8, 9, (rows, 3), device=DEV, generator=g).bfloat16()
    out = P.camera_token_logprobs(z, top_n=n, entropy=False)
    idx, lp = out["top_idx"], out["top_logprob"]
    torch.cuda.synchronize()
    step = 1 << 20
    for r in list(range(0, rows, step)):
        zc = z[r:r + step].float()
        want = torch.log_softmax(zc, 1)
        order = torch.sort(zc, dim=1, descending=True, stable=True).indices
        assert torch.equal(idx[r:r + step, :3].long(), order), r
        assert (lp[r:r + step, :3] - want.gather(1, order)).abs().max() <= 1e-5, r
        assert (idx[r:r + step, 3:] == -1).all() and (lp[r:r + step, 3:] == -float("inf")).all(), r
