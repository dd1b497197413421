"""The limit of the waits between CTAs that share a row of logits.  With the shortest limit (1 us) a row's results are
right or NaN, every call returns, and calls with the ordinary limit are right again afterwards."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


@pytest.fixture
def short(P):
    default = P.camera_get_wait_limit_ns()

    class Limit:
        def __enter__(self):
            P.camera_set_wait_limit_ns(1000)

        def __exit__(self, *exc):
            torch.cuda.synchronize()
            P.camera_set_wait_limit_ns(default)
    yield Limit()
    P.camera_set_wait_limit_ns(default)


def same_or_nan(got, want):
    """Element by element; returns how many are NaN."""
    nan = got.isnan()
    assert torch.equal(got[~nan], want[~nan])
    return int(nan.sum())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_alternatives_of_which_a_part_is_late(P, short, dtype):
    """The second half of each row is one value, whose ties take the CTAs that read it hundreds of microseconds to sort out
    while the first one waits."""
    rows, vocab, n = 30, 151936, 100
    g = torch.Generator(device=DEV).manual_seed(1)
    z = torch.randn(rows, vocab, device=DEV, generator=g)
    z[:, vocab // 2:] = 6.0
    z = z.to(dtype)
    targets = torch.randint(0, vocab, (rows,), device=DEV, generator=g)
    want = P.camera_token_logprobs(z, targets, top_n=n)
    ran_out = 0
    for _ in range(5):
        with short:
            got = P.camera_token_logprobs(z, targets, top_n=n)
        same_or_nan(got["logprob"], want["logprob"])
        same_or_nan(got["entropy"], want["entropy"])
        ran_out += same_or_nan(got["top_logprob"], want["top_logprob"])
        nan = got["top_logprob"].isnan()
        assert (got["top_idx"][nan] == -1).all() and torch.equal(got["top_idx"][~nan], want["top_idx"][~nan])
        assert torch.equal(nan.all(1), nan.any(1))           # a row has all of its alternatives or none
    assert ran_out > 0                                       # or the test has shown nothing
    again = P.camera_token_logprobs(z, targets, top_n=n)
    assert all(torch.equal(again[k], want[k]) for k in want)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("rows,vocab", [(3, 151936), (37, 60001), (700, 110001)])
def test_distillation(P, short, tail, rows, vocab):
    g = torch.Generator(device=DEV).manual_seed(2)
    z = (torch.randn(rows, vocab, device=DEV, generator=g) * 2).bfloat16()
    z[1, : vocab // 2] = -float("inf")
    z[0] = -60000.0                                          # the careful walk
    idx = torch.stack([torch.randperm(vocab, device=DEV, generator=g)[:64] for _ in range(rows)]).int()
    lp = torch.log_softmax(torch.randn(rows, 64, device=DEV, generator=g), 1) - 0.1
    d_loss = torch.ones(rows, device=DEV)
    call = lambda: P.camera_distill_step(z, idx, lp, d_loss, tail=tail)
    want = call()
    for _ in range(5):
        with short:
            got = call()
            f = P.camera_distill_forward(z, idx, lp, tail=tail)
        for a, b in zip(got, want):
            same = (a == b) | (a.isnan() & b.isnan())
            assert (same | a.isnan()).all()
        f_same = (f["loss"] == want[0]) | f["loss"].isnan()
        assert f_same.all()
    again = call()
    for a, b in zip(again, want):
        assert torch.equal(a.nan_to_num(nan=123.0), b.nan_to_num(nan=123.0))
