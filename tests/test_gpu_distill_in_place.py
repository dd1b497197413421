"""camera_distill_backward and camera_distill_step with the gradient in the logits' room: the same bits as beside them."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("rows,vocab,k,pad,shift", [
    (1, 5, 3, 0, 0), (1, 151936, 128, 0, 0),            # a row in parts
    (3, 60001, 64, 7, 1), (37, 32003, 20, 5, 3),        # rows in parts, several of them, unaligned
    (321, 110001, 40, 7, 0), (700, 1009, 64, 0, 2)])    # more rows than run at one time
def test_in_place(P, dtype, tail, rows, vocab, k, pad, shift):
    g = torch.Generator(device=DEV).manual_seed(rows + vocab)
    buf = torch.zeros(rows * (vocab + pad) + shift, dtype=dtype, device=DEV)
    view = lambda b: b[shift:].view(rows, vocab + pad)[:, :vocab]
    z = view(buf)
    z.copy_(torch.randn(rows, vocab, device=DEV, generator=g) * 3)
    idx = torch.stack([torch.randperm(vocab, device=DEV, generator=g)[:k] for _ in range(rows)]).int()
    lp = torch.log_softmax(torch.randn(rows, k, device=DEV, generator=g), 1) - 0.1
    d_loss = torch.rand(rows, device=DEV, generator=g) + 0.5
    if rows > 2:
        d_loss[1::5] = 0.0
    f = P.camera_distill_forward(z, idx, lp, temperature=1.2, tail=tail)
    beside = P.camera_distill_backward(z, idx, lp, d_loss, f["lse"], f.get("log_tail"), temperature=1.2, tail=tail)
    _, step = P.camera_distill_step(z, idx, lp, d_loss, temperature=1.2, tail=tail)
    for name, want in (("backward", beside), ("step", step)):
        again = buf.clone()
        z2 = view(again)
        if name == "backward":
            got = P.camera_distill_backward(z2, idx, lp, d_loss, f["lse"], f.get("log_tail"), temperature=1.2, tail=tail, d_logits=z2)
        else:
            _, got = P.camera_distill_step(z2, idx, lp, d_loss, temperature=1.2, tail=tail, d_logits=z2)
        assert got is z2 and torch.equal(z2, want), name
        # what lies between the rows is left alone
        if pad:
            gaps = lambda b: b[shift:].view(rows, vocab + pad)[:, vocab:]
            assert torch.equal(gaps(again), gaps(buf))
        assert torch.equal(again[:shift], buf[:shift])
