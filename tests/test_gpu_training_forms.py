"""The operators around a layer's experts in the forms their kernels take that sizes of whole 16 bytes or odd widths do not reach:
rows read two elements at a time, several packs a thread in combine, long rows whose weight gradient is asked for alone.
References and tolerances are those of test_gpu_moe.py and test_gpu_norm.py.
"""
import pytest
import torch

from test_gpu_moe import U, close, gathered, matrix, routing, sort_ref
from test_gpu_norm import backward_ref, check, forward_ref, rows_of

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def sorted_rows(P, g, tokens, k, experts, d, dtype, pad, first):
    idx = routing(g, tokens, k, experts, 0.1)
    rows, offsets, pairs = sort_ref(idx, experts)
    x = matrix(g, tokens, d, dtype, pad, first)
    out = matrix(g, tokens * k + 1, d, dtype, pad, first)
    before = out.clone()
    r = P.camera_moe_dispatch(x, idx, experts, out=out)
    assert torch.equal(r["rows"].cpu(), rows) and torch.equal(r["offsets"].cpu(), offsets)
    n = len(pairs)
    assert torch.equal(out[:n], x[torch.tensor(pairs, dtype=torch.long, device=DEV) // k]) and torch.equal(out[n:], before[n:])
    return rows.to(DEV)


def there_and_back(P, tokens, k, experts, d, dtype, pad, first):
    g = torch.Generator(device=DEV).manual_seed(tokens + 31 * k + d)
    rows = sorted_rows(P, g, tokens, k, experts, d, dtype, pad, first)
    n = tokens * k
    ys, add, dy = (matrix(g, m, d, dtype, pad, first) for m in (n, tokens, tokens))
    w = torch.rand((tokens, k), device=DEV, generator=g) - 0.3
    got, ok = gathered(rows, n, ys)
    for weights, extra in ((w, add), (None, None)):
        wd = ok.double() if weights is None else weights.double() * ok
        terms = got * wd[:, :, None]
        want, size = terms.sum(1), terms.abs().sum(1)
        if extra is not None:
            want, size = want + extra.double(), size + extra.double().abs()
        close(P.camera_moe_combine(ys, rows, weights, add=extra), want, (k + 2) * U * size, dtype)
    close(P.camera_moe_dispatch_backward(ys, rows, add=add), got.sum(1) + add.double(), (k + 2) * U * (got.abs().sum(1) + add.double().abs()), dtype)
    for dots in (True, False):
        out = matrix(g, n, d, dtype, pad, first)
        before = out.clone()
        r = P.camera_moe_combine_backward(dy, ys, rows, w, out=out, want_weights=dots)
        named = torch.zeros(n, dtype=torch.bool, device=DEV)
        named[rows[ok].long()] = True
        assert torch.equal(out[~named], before[~named])
        full = (w.double() * ok)[:, :, None] * dy.double()[:, None, :]
        close(out[rows[ok].long()], full[ok], U * full[ok].abs(), dtype)
        if dots:
            prod = got * dy.double()[:, None, :]
            close(r["weights"], prod.sum(2), (d + 8) * U * prod.abs().sum(2), F32)
            assert not r["weights"][~ok].any()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tokens,k,experts,d,pad,first", [
    (33, 2, 8, 34, 0, 0), (65, 6, 64, 130, 0, 0), (300, 16, 200, 2, 0, 0), (5, 1, 4, 2050, 0, 0), (200, 3, 16, 64, 2, 2), (64, 8, 64, 1024, 2, 0),
    (777, 1, 61, 1002, 0, 0), (777, 2, 61, 1002, 2, 2), (777, 3, 61, 1002, 0, 2), (777, 4, 61, 1002, 4, 0), (777, 8, 61, 1002, 0, 0), (320, 5, 8, 4098, 0, 0)])
def test_tokens_by_two_elements(P, tokens, k, experts, d, pad, first, dtype):
    there_and_back(P, tokens, k, experts, d, dtype, pad, first)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("k", [1, 2, 3, 4])
@pytest.mark.parametrize("tokens,d", [(3000, 1024), (1500, 2056), (400, 8200), (1001, 1001)])
def test_tokens_of_several_packs_a_thread(P, tokens, d, k, dtype):
    there_and_back(P, tokens, k, 32, d, dtype, 0, 0)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("rows,d,pad,first", [
    (3, 8200, 0, 0), (700, 8200, 0, 0), (9, 16384, 0, 0), (400, 16384, 0, 0), (5, 16392, 0, 0), (310, 16392, 0, 0), (2, 32767, 0, 0), (170, 32767, 0, 0),
    (3, 32768, 0, 0), (300, 32768, 0, 0), (300, 8704, 1, 0), (20, 17024, 1, 1), (160, 20002, 0, 0), (40, 9002, 2, 2), (30, 602, 0, 2), (2000, 130, 2, 0)])
def test_weight_gradients_alone(P, rows, d, pad, first, rms, dtype):
    g = torch.Generator(device=DEV).manual_seed(rows + d)
    x, dy = rows_of(g, rows, d, dtype, pad, first, shift=0.3), rows_of(g, rows, d, dtype, pad, first, 0.1)
    ds = rows_of(g, rows, d, dtype, pad, first, 0.1)
    w = 1 + 0.2 * torch.randn(d, device=DEV, generator=g)
    out = P.camera_norm_forward(x, w, rms=rms)
    check(out, forward_ref(x, w, None, 1e-6, rms, dtype), ["y", "rstd"])
    ws = P.alloc_workspace(P.camera_norm_backward_workspace_bytes(rows, d), DEV).fill_(255)
    grads = P.camera_norm_backward(dy, x, out["rstd"], out.get("mean"), w, d_sum=ds, workspace=ws)
    ref = backward_ref(dy, x, out.get("mean"), out["rstd"], w, ds, dtype, rows)
    check(grads, ref, ["x", "weight"])
    only = P.camera_norm_backward(dy, x, out["rstd"], out.get("mean"), w, want_x=False, want_weight=False, want_bias=True, workspace=ws.fill_(255))
    assert set(only) == {"bias"}
    check(only, ref, ["bias"])


def test_the_weight_gradient_of_more_than_2_31_elements(P):
    rows, d = 262145, 8208
    x = torch.empty(rows, d, dtype=BF, device=DEV).normal_()
    dy = torch.empty(rows, d, dtype=BF, device=DEV).normal_()
    rstd = P.camera_norm_forward(x, rms=True)["rstd"]
    grads = P.camera_norm_backward(dy, x, rstd)
    want, size = torch.zeros(d, dtype=torch.float64, device=DEV), torch.zeros(d, dtype=torch.float64, device=DEV)
    for a in range(0, rows, 8192):
        part = dy[a:a + 8192].double() * (x[a:a + 8192].double() * rstd[a:a + 8192, None].double())
        want += part.sum(0)
        size += part.abs().sum(0)
    assert ((grads["weight"].double() - want).abs() <= 2 * (rows + 68) * U * size).all()
    for part in (slice(0, 500), slice(rows - 500, rows)):
        ref = backward_ref(dy[part], x[part], None, rstd[part], None, None, BF, 500)
        check({"x": grads["x"][part]}, ref, ["x"])
    del x, dy, grads
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale", [1e17, 1e-17])
def test_norms_of_large_and_small_rows(P, scale, dtype):
    """Near the ends of what squares in fp32 hold; eps does not enter."""
    g = torch.Generator(device=DEV).manual_seed(1)
    for rows, d in ((700, 1000), (5, 33), (300, 9000)):
        x, dy = rows_of(g, rows, d, dtype).clamp_(-3, 3).mul_(scale / 3), rows_of(g, rows, d, dtype, scale=0.1)
        w = 1 + 0.2 * torch.randn(d, device=DEV, generator=g)
        for rms in (False, True):
            out = P.camera_norm_forward(x, w, eps=0.0, rms=rms)
            check(out, forward_ref(x, w, None, 0.0, rms, dtype), ["y", "rstd"] + ([] if rms else ["mean"]))
            grads = P.camera_norm_backward(dy, x, out["rstd"], out.get("mean"), w, want_bias=True)
            check(grads, backward_ref(dy, x, out.get("mean"), out["rstd"], w, None, dtype, rows), ["x", "weight", "bias"])
