"""Calls from several host threads at once, of shapes that take different amounts of shared memory."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def test_threads(P):
    g = torch.Generator(device=DEV).manual_seed(1)
    shapes = [(2, 20000 * (i + 1)) for i in range(12)]
    work = []
    for rows, vocab in shapes:
        z = torch.randn(rows, vocab, device=DEV, generator=g)
        idx = torch.stack([torch.randperm(vocab, device=DEV, generator=g)[:16] for _ in range(rows)]).int()
        lp = torch.log_softmax(torch.randn(rows, 16, device=DEV, generator=g), 1) - 0.1
        work.append((z, idx, lp, torch.ones(rows, device=DEV)))
    torch.cuda.synchronize()
    gate, out, errors = threading.Barrier(len(work)), {}, []

    def call(i, n):
        stream = torch.cuda.Stream()
        try:
            gate.wait()
            for k in range(n):
                z, idx, lp, d_loss = work[(i + k) % len(work)]
                out[i, k] = P.camera_distill_step(z, idx, lp, d_loss, tail=True, stream=stream) + \
                    (P.camera_token_logprobs(z, top_n=10 * (i + 1), stream=stream)["top_idx"],)
            stream.synchronize()
        except Exception as e:            # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=call, args=(i, 24)) for i in range(len(work))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for (i, k), (loss, grad, top) in out.items():
        z, idx, lp, d_loss = work[(i + k) % len(work)]
        want = P.camera_distill_step(z, idx, lp, d_loss, tail=True) + (P.camera_token_logprobs(z, top_n=10 * (i + 1))["top_idx"],)
        assert torch.equal(loss, want[0]) and torch.equal(grad, want[1]) and torch.equal(top, want[2])
