"""Layer norm and root-mean-square norm, forward and backward, against float64 on the same stored values.

Tolerances, derived before the first run, with u = 2^-24 (half a step of fp32) and e = half a step of the dtype.  A row's sum
passes at most 32 additions in a thread, 5 in a warp, 32 over warps and a division: N = 72 roundings, so a mean of v is off by
at most N u mean|v|.  First-order effects in y: the mean's error times s |w|, a relative error of s of at most (N + 4) u plus
the mean's error over the deviation, three roundings of the product, one of the sum with the bias, one to the dtype.  In dx:
those of g, h (2 each) and of the two means.  Sums over rows pass at most n_rows + 64 additions.  All bounds are doubled for
the terms of second order.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U, N = 2.0 ** -24, 72
BF, F32 = torch.bfloat16, torch.float32


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def rows_of(g, rows, d, dtype, pad=0, first=0, scale=1.0, shift=0.0):
    """A [rows, d] matrix of pitch d + pad that starts `first` elements into its storage."""
    buf = torch.zeros(rows * (d + pad) + first + 16, dtype=dtype, device=DEV)
    m = buf[first:first + rows * (d + pad)].view(rows, d + pad)[:, :d]
    m.copy_(torch.randn(rows, d, device=DEV, generator=g) * scale + shift)
    return m


def forward_ref(z, w, b, eps, rms, dtype):
    z = z.double()
    w = torch.ones(z.shape[1], device=DEV, dtype=torch.float64) if w is None else w.double()
    b = torch.zeros_like(w) if b is None else b.double()
    mu = torch.zeros_like(z[:, 0]) if rms else z.mean(1)
    c = z - mu[:, None]
    s = (c.pow(2).mean(1) + eps).rsqrt()
    y = c * s[:, None] * w + b
    d_mu = torch.zeros_like(mu) if rms else N * U * z.abs().mean(1)
    rel = (N + 6) * U + d_mu * s
    tol = (y - b).abs() * (rel[:, None] + 3 * U) + (d_mu * s)[:, None] * w.abs() + U * y.abs()
    return {"mean": (mu, 2 * d_mu + U * mu.abs()), "rstd": (s, 2 * rel * s),
            "y": (y, 2 * tol + half_step(dtype) * (y.abs() + 2 * tol) + 1e-38)}


def backward_ref(dy, z, mean, rstd, w, d_sum, dtype, rows):
    dy, z, s = dy.double(), z.double(), rstd.double()[:, None]
    w = torch.ones(z.shape[1], device=DEV, dtype=torch.float64) if w is None else w.double()
    rms = mean is None
    c = z if rms else z - mean.double()[:, None]
    h, g = c * s, dy * w
    m1 = torch.zeros_like(s) if rms else g.mean(1, keepdim=True)
    m2 = (g * h).mean(1, keepdim=True)
    dx = s * (g - m1 - h * m2)
    t1 = torch.zeros_like(s) if rms else (N + 1) * U * g.abs().mean(1, keepdim=True)
    t2 = (N + 4) * U * (g * h).abs().mean(1, keepdim=True)
    tol = s * (4 * U * g.abs() + 3 * U * m1.abs() + 6 * U * (h * m2).abs() + t1 + h.abs() * t2) + U * dx.abs()
    if d_sum is not None:
        dx = dx + d_sum.double()
        tol = tol + U * dx.abs()
    n = (rows + 64) * U
    dw, db = (dy * h).sum(0), dy.sum(0)
    return {"x": (dx, 2 * tol + half_step(dtype) * (dx.abs() + 2 * tol) + 1e-38), "weight": (dw, 2 * (n + 4 * U) * (dy * h).abs().sum(0)),
            "bias": (db, 2 * n * dy.abs().sum(0))}


def check(got, ref, names):
    for name in names:
        want, tol = ref[name]
        err = (got[name].double() - want).abs()
        bad = ~(err <= tol)
        assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst {float((err / tol).max()):.2f} of it"


def run(P, rows, d, dtype, rms, residual, bias, w_dtype, pad=0, first=0, seed=0, shift=0.3, eps=1e-6, weight=True):
    g = torch.Generator(device=DEV).manual_seed(seed + rows + d)
    x = rows_of(g, rows, d, dtype, pad, first, shift=shift)
    r = rows_of(g, rows, d, dtype, pad, first, 0.5) if residual else None
    w = (1 + 0.2 * torch.randn(d, device=DEV, generator=g)).to(w_dtype) if weight else None
    b = (0.1 * torch.randn(d, device=DEV, generator=g)).to(w_dtype) if bias else None
    out = P.camera_norm_forward(x, w, b, residual=r, eps=eps, rms=rms)
    z = x
    if residual:
        z = out["sum"]
        assert torch.equal(z, (x.float() + r.float()).to(dtype))
    assert ("mean" in out) == (not rms)
    check(out, forward_ref(z, w, b, eps, rms, dtype), ["y", "rstd"] + ([] if rms else ["mean"]))
    dy = rows_of(g, rows, d, dtype, pad, first, 0.1)
    ds = rows_of(g, rows, d, dtype, pad, first, 0.1) if residual else None
    ws = P.alloc_workspace(P.camera_norm_backward_workspace_bytes(rows, d), DEV).fill_(255)
    grads = P.camera_norm_backward(dy, z, out["rstd"], out.get("mean"), w, d_sum=ds, want_bias=True, workspace=ws)
    check(grads, backward_ref(dy, z, out.get("mean"), out["rstd"], w, ds, dtype, rows), ["x", "weight", "bias"])
    return x, r, w, b, dy, ds, out, grads


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("rows,d,pad,first", [
    (1, 1, 0, 0), (1, 8, 0, 0), (3, 7, 0, 0), (2, 16, 0, 0), (5, 33, 2, 1), (1, 3584, 0, 0), (9, 256, 8, 8), (300, 264, 0, 0),
    (17, 1000, 0, 0), (17, 1000, 1, 0), (64, 1001, 7, 0), (129, 2048, 0, 4), (129, 2048, 0, 1), (700, 512, 16, 0), (2500, 72, 0, 0),
    (310, 3584, 0, 0), (40, 8192, 0, 0), (40, 8200, 0, 0), (7, 16384, 0, 0), (5, 16392, 0, 0), (3, 32768, 0, 0), (3, 32767, 0, 0),
    (5000, 24, 0, 0), (1001, 8191, 0, 0)])
def test_sizes_strides_and_types(P, rows, d, pad, first, rms, dtype):
    run(P, rows, d, dtype, rms, residual=(rows + d) % 2 == 0, bias=not rms, w_dtype=F32 if d % 3 else dtype, pad=pad, first=first)


def test_without_weights(P):
    run(P, 33, 520, BF, False, False, False, BF, weight=False)
    run(P, 33, 521, F32, True, True, False, F32, weight=False)


def test_a_large_mean_costs_the_deviation_nothing(P):
    """Rows around 300 with a deviation of 1: a variance taken as a difference of squares would lose 17 bits."""
    run(P, 50, 1024, F32, False, False, True, F32, shift=300.0)
    run(P, 50, 1023, F32, False, False, True, F32, shift=-300.0)


def test_rows_without_variance(P):
    x = torch.full((4, 96), 2.5, device=DEV)
    y = P.camera_norm_forward(x, bias=torch.full((96,), 0.25, device=DEV), eps=1e-5)
    assert (y["y"] == 0.25).all() and torch.allclose(y["rstd"], torch.full((4,), 1e-5 ** -0.5, device=DEV), rtol=1e-6)
    zero = P.camera_norm_forward(torch.zeros(3, 40, dtype=BF, device=DEV), rms=True)
    assert not zero["y"].any()
    assert torch.isnan(P.camera_norm_forward(torch.zeros(3, 40, device=DEV), rms=True, eps=0.0)["y"]).all()


def test_a_nan_or_infinity_stays_in_its_row(P):
    for d in (1024, 1023):
        x = torch.randn(100, d, device=DEV).bfloat16()
        clean = P.camera_norm_forward(x, rms=False)
        x[3, 5], x[50, 7] = float("nan"), float("inf")
        y = P.camera_norm_forward(x, rms=False)
        keep = torch.ones(100, dtype=torch.bool, device=DEV)
        keep[3] = keep[50] = False
        assert torch.isnan(y["y"][3]).all() and torch.isnan(y["y"][50]).any()
        assert torch.equal(y["y"][keep], clean["y"][keep]) and torch.equal(y["rstd"][keep], clean["rstd"][keep])


def test_no_rows(P):
    x = torch.zeros(0, 64, dtype=BF, device=DEV)
    out = P.camera_norm_forward(x, residual=x)
    assert out["y"].shape == (0, 64) and out["sum"].shape == (0, 64)
    grads = P.camera_norm_backward(x, x, out["rstd"], out["mean"], want_bias=True)
    assert grads["x"].shape == (0, 64) and not grads["weight"].any() and not grads["bias"].any()


@pytest.mark.parametrize("d", [2048, 2047])
def test_results_may_take_the_inputs_room(P, d):
    x, r, w, b, dy, ds, out, grads = run(P, 600, d, BF, False, True, True, BF)
    x2, r2 = x.clone(), r.clone()
    a = P.camera_norm_forward(x2, w, b, residual=r2, out={"y": x2, "sum": r2})
    assert torch.equal(x2, out["y"]) and torch.equal(r2, out["sum"]) and torch.equal(a["rstd"], out["rstd"])
    for k in range(3):
        dy2, ds2, z2 = dy.clone(), ds.clone(), out["sum"].clone()
        got = P.camera_norm_backward(dy2, z2, out["rstd"], out["mean"], w, d_sum=ds2, out=(dy2, ds2, z2)[k])
        assert torch.equal(got["x"], grads["x"]) and torch.equal(got["weight"], grads["weight"])


def test_parts_can_be_asked_for_and_repeat_bit_for_bit(P):
    x, r, w, b, dy, ds, out, grads = run(P, 1300, 776, F32, True, True, False, F32)
    z = out["sum"]
    only = P.camera_norm_backward(dy, z, out["rstd"], None, w, d_sum=ds, want_weight=False)
    assert set(only) == {"x"} and torch.equal(only["x"], grads["x"])
    weights = P.camera_norm_backward(dy, z, out["rstd"], None, w, want_x=False)
    assert set(weights) == {"weight"} and torch.equal(weights["weight"], grads["weight"])
    assert set(P.camera_norm_forward(x, w, rms=True, stats=False)) == {"y"}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = P.camera_norm_backward(dy, z, out["rstd"], None, w, d_sum=ds, want_bias=True, stream=side)
    side.synchronize()
    for k, t in grads.items():
        assert torch.equal(again[k], t), k


def test_a_workspace_serves_every_smaller_call(P):
    for d in (40, 264, 1000, 3584, 12000):
        sizes = [P.camera_norm_backward_workspace_bytes(n, d) for n in range(1, 4000, 7)]
        assert sizes == sorted(sizes)
    ws = P.alloc_workspace(P.camera_norm_backward_workspace_bytes(3000, 264), DEV)
    for n in (1, 2, 150, 299, 1199, 3000):
        z, dy = torch.randn(n, 264, device=DEV), torch.randn(n, 264, device=DEV)
        s = torch.ones(n, device=DEV)
        a = P.camera_norm_backward(dy, z, s, workspace=ws, want_bias=True)
        check(a, backward_ref(dy, z, None, s, None, None, F32, n), ["x", "weight", "bias"])


def test_gradient_against_differences(P):
    """Central differences of L = <dy, y> in float64 along random directions (step 1e-4, error of order 1e-8)."""
    for rms in (False, True):
        x, r, w, b, dy, ds, out, grads = run(P, 20, 88, F32, rms, False, not rms, F32)
        ref = backward_ref(dy, x, out.get("mean"), out["rstd"], w, None, F32, 20)
        loss = lambda z, w_: float((dy.double() * forward_ref(z, w_, b, 1e-6, rms, F32)["y"][0]).sum())
        for name, leaf in (("x", x), ("weight", w)):
            v = torch.randn(leaf.shape, device=DEV, dtype=torch.float64)
            at = [leaf.double() + k * 1e-4 * v for k in (1, -1)]
            want = (loss(at[0], w) - loss(at[1], w) if name == "x" else loss(x, at[0]) - loss(x, at[1])) / 2e-4
            got = float((grads[name].double() * v).sum())
            # rstd and mean enter rounded to fp32: 2^-24 of terms of the size of the result's parts
            tol = float((ref[name][1] * v.abs()).sum()) + 1e-5
            assert abs(got - want) <= tol, (rms, name, got, want, tol)


def test_a_captured_pass_replays_with_new_inputs(P):
    x, dy = torch.randn(500, 1024, device=DEV).bfloat16(), torch.randn(500, 1024, device=DEV).bfloat16()
    w = torch.randn(1024, device=DEV)
    ws = P.alloc_workspace(P.camera_norm_backward_workspace_bytes(500, 1024), DEV)

    def both():
        f = P.camera_norm_forward(x, w, rms=True)
        return f["y"], P.camera_norm_backward(dy, x, f["rstd"], None, w, workspace=ws)
    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, grads = both()
    x.copy_(torch.randn(500, 1024, device=DEV))
    graph.replay()
    torch.cuda.synchronize()
    y2, g2 = both()
    assert torch.equal(y, y2) and torch.equal(grads["x"], g2["x"]) and torch.equal(grads["weight"], g2["weight"])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,d,pad,first", [
    (1, 64, 1, 1), (900, 64, 3, 0), (2000, 264, 1, 1), (600, 2048, 1, 0), (333, 8192, 1, 3), (300, 8704, 1, 0), (20, 17024, 1, 1), (3, 32768, 1, 0)])
def test_rows_off_their_boundaries(P, rows, d, pad, first, dtype):
    """What is read lies on odd elements, what is written on boundaries of 16 bytes; weights at an odd place too."""
    for rms in (False, True):
        x, r, w, b, dy, ds, out, grads = run(P, rows, d, dtype, rms, True, not rms, F32, pad=pad, first=first)
        off = torch.empty(d + 1, device=DEV)[1:]
        off.copy_(w)
        again = P.camera_norm_forward(x, off, b, residual=r, rms=rms)
        assert torch.equal(again["y"], out["y"])
        tight = P.camera_norm_forward(x.contiguous(), w, b, residual=r.contiguous(), rms=rms)
        check(out | tight, forward_ref(out["sum"], w, b, 1e-6, rms, dtype), ["y", "rstd"])
        g2 = P.camera_norm_backward(dy, out["sum"], out["rstd"], out.get("mean"), off, d_sum=ds, want_bias=True)
        for k in grads:
            assert torch.equal(g2[k], grads[k]), k


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,d", [(20000, 600), (20000, 602), (20000, 601), (9000, 96), (9000, 97), (7000, 1200), (40000, 1)])
def test_many_groups_of_a_cta_share_their_sums(P, rows, d, dtype):
    for bias in (False, True):
        x, r, w, b, dy, ds, out, grads = run(P, rows, d, dtype, True, False, False, F32)
        only = P.camera_norm_backward(dy, x, out["rstd"], None, w, want_x=False, want_weight=not bias, want_bias=bias)
        for k in only:
            assert torch.equal(only[k], grads[k]), k


@pytest.mark.parametrize("rows,d", [(1, 64), (3, 1000), (1, 3584), (2, 32768), (16, 256)])
def test_few_rows_and_gradients_at_odd_places(P, rows, d):
    """One CTA writes the weights' gradients itself, unless they lie off 16-byte boundaries; nothing around them is written."""
    import ctypes as C
    x, r, w, b, dy, ds, out, grads = run(P, rows, d, F32, False, False, True, F32)
    ws = P.alloc_workspace(P.camera_norm_backward_workspace_bytes(rows, d), DEV)
    from paper_2508_02322_b200.binding import CAMERA_F32, camera_norm_t
    n = camera_norm_t(x.data_ptr(), d, rows, CAMERA_F32, d, w.data_ptr(), None, CAMERA_F32, 0.0, 0)
    for at in (0, 1, 3):
        dw, db = torch.full((d + 8,), 7.0, device=DEV), torch.full((d + 8,), 7.0, device=DEV)
        assert P.lib.camera_norm_backward(C.byref(n), dy.data_ptr(), d, out["mean"].data_ptr(), out["rstd"].data_ptr(), None, 0, None, 0,
                                          dw[at:].data_ptr(), db[at:].data_ptr(), ws.data_ptr(), ws.numel(),
                                          torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(dw[at:at + d], grads["weight"]) and torch.equal(db[at:at + d], grads["bias"])
        assert (dw[:at] == 7.0).all() and (dw[at + d:] == 7.0).all() and (db[:at] == 7.0).all() and (db[at + d:] == 7.0).all()
