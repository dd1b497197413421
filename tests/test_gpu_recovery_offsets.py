"""Tensors of more than 2^31 elements: the kept products and activations of a feed-forward block, rows of logits."""
import pytest
import torch

from _distill_ref import close

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def test_feed_forward_block(P):
    """Rounding to bf16 (2^-9) of the gated product, dG and dU and of the result: errors of about 2^-9 of the typical size of
    a result; 2^-5 of it on single elements leaves room, a wrong row is off by all of it."""
    T, D, F = 56000, 64, 20001                          # 2 * pitch * T = 2.25e9
    g = torch.Generator(device=DEV).manual_seed(1)
    r = lambda *s: torch.randn(s, device=DEV, generator=g)
    ffn = P.Ffn((r(F, D) * 0.125).bfloat16(), (r(F, D) * 0.125).bfloat16(), (r(D, 20008) * 0.01).bfloat16(), d_ff=F)
    x, dy = r(T, D).bfloat16(), (r(T, D) * 0.01).bfloat16()
    saved = P.alloc_workspace(P.camera_ffn_saved_bytes(ffn, T), DEV)
    ws = P.alloc_workspace(P.camera_ffn_workspace_bytes(ffn, T, backward=True), DEV)
    y = P.camera_ffn_forward(ffn, x, saved=saved, workspace=ws)
    grads = P.camera_ffn_backward(ffn, x, dy, saved, workspace=ws)
    assert P.camera_read_status(ws) == 0
    wg, wu, wd = ffn.w_gate.double(), ffn.w_up.double(), ffn.w_down[:, :F].double()
    total = {n: torch.zeros(s, device=DEV, dtype=torch.float64) for n, s in (("w_gate", (F, D)), ("w_up", (F, D)), ("w_down", (D, F)))}
    near = lambda a, b: float((a.double() - b).abs().max() / b.square().mean().sqrt())
    for t in range(0, T, 4000):
        xd, dyd = x[t:t + 4000].double(), dy[t:t + 4000].double()
        a, u, dh = xd @ wg.t(), xd @ wu.t(), dyd @ wd
        s = torch.sigmoid(a)
        h, du, dg = a * s * u, dh * a * s, dh * u * s * (1 + a * (1 - s))
        assert near(y[t:t + 4000], h @ wd.t()) < 2.0 ** -5, t
        assert near(grads["x"][t:t + 4000], dg @ wg + du @ wu) < 2.0 ** -5, t
        total["w_gate"] += dg.t() @ xd
        total["w_up"] += du.t() @ xd
        total["w_down"] += dyd.t() @ h
    for name, want in total.items():
        assert near(grads[name][:, :F] if name == "w_down" else grads[name], want) < 2.0 ** -5, name


@pytest.mark.parametrize("tail", [False, True])
def test_rows_of_logits(P, tail):
    rows, vocab, k = 15001, 151936, 8                   # 2.28e9 logits
    g = torch.Generator(device=DEV).manual_seed(2)
    some = torch.randn(7, vocab, device=DEV, generator=g).bfloat16()
    z = some.repeat((rows + 6) // 7, 1)[:rows]
    idx = (torch.arange(k, device=DEV, dtype=torch.int32) * 1000 + 5).expand(rows, -1).contiguous()
    lp = torch.full((rows, k), -2.5, device=DEV)
    d_loss = torch.ones(rows, device=DEV)
    top = P.camera_token_logprobs(z, torch.full((rows,), 17, device=DEV), top_n=3)
    loss, grad = P.camera_distill_step(z, idx, lp, d_loss, tail=tail)
    f = P.camera_distill_forward(z, idx, lp, tail=tail)
    back = P.camera_distill_backward(z, idx, lp, d_loss, f["lse"], f.get("log_tail"), tail=tail)
    # against the first rows, which the other tests hold to float64; the rows repeat
    few = P.camera_distill_step(some, idx[:7], lp[:7], d_loss[:7], tail=tail)
    close(loss[:7], few[0].double().cpu().numpy(), 1e-4)
    for t in (loss, f["loss"], top["logprob"], top["entropy"], top["top_idx"], top["top_logprob"]):
        assert torch.equal(t[7:], t[: rows - 7])
    for t in (grad, back):
        assert (t[:7].double() - few[1].double()).abs().max() <= 1e-4
        for r in range(7, rows, 700):
            assert torch.equal(t[r:r + 700], t[r - 7: r - 7 + 700][: t[r:r + 700].shape[0]]), r
