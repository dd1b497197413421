"""The gated feed-forward block, forward and backward, against float64 on the same stored values.

Tolerances, derived before the first run.  The kernels multiply bf16 exactly and add in fp32 (error below 2^-18 of the
sum of magnitudes for the sizes here), and round to bf16 (relative error u = 2^-9) at these places: the gated product h,
the kept products g and u, their gradients dg and du, and the result.  First-order errors of the intermediate values are
  h:  u |h| (forward);  u (|h| + |f'(g) g u| + |h|) (recomputed from rounded g and u)      with f = SiLU
  du: u |dh| (|f(g)| + |f'(g) g|),   dg: u |dh| |u| (2 |f'(g)| + |f''(g) g|)
and they enter a result as a sum over independent roundings, so the result's error is its own rounding u |r| plus a sum
whose standard deviation is at most E = sqrt(sum (error * factor)^2).  The bound is 2 u |r| + 6 E + 2^-17 sqrt(sum
(value * factor)^2): six standard deviations leave one failure in 10^9 elements, and half the bound already has slack of
sqrt(3), a rounding error being uniform.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -9


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def make(T, D, F, ld, seed=0, x_scale=1.0, w_scale=0.05):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(s, device=DEV, generator=g)
    return ((r(T, D) * x_scale).bfloat16(), (r(F, D) * w_scale).bfloat16(), (r(F, D) * w_scale).bfloat16(),
            (r(D, ld) * w_scale).bfloat16(), (r(T, D) * 0.1).bfloat16())


def reference(x, wg, wu, wd, dy, F):
    """Results in float64 and the bound of each (see above)."""
    x, wg, wu, wd, dy = (t.double() for t in (x, wg, wu, wd[:, :F], dy))
    g, u = x @ wg.t(), x @ wu.t()
    s = torch.sigmoid(g)
    f, f1 = g * s, s * (1 + g * (1 - s))
    f2 = s * (1 - s) * (2 + g * (1 - 2 * s))
    h, dh = f * u, dy @ wd
    du, dg = dh * f, dh * u * f1
    e_h = U * (2 * h.abs() + (f1 * g * u).abs())
    e_du = U * dh.abs() * (f.abs() + (f1 * g).abs()) + U * du.abs()
    e_dg = U * (dh * u).abs() * (2 * f1.abs() + (f2 * g).abs()) + U * dg.abs()
    sq = lambda a, b: (a.square() @ b.square()).sqrt()
    bound = lambda r, e, v: 2 * U * r.abs() + 6 * e + 2.0 ** -17 * v + 1e-30
    y, dx = h @ wd.t(), dg @ wg + du @ wu
    out = {"y": (y, bound(y, sq(U * h, wd.t()), sq(h, wd.t()))),
           "x": (dx, bound(dx, (sq(e_dg, wg).square() + sq(e_du, wu).square()).sqrt(), sq(dg, wg) + sq(du, wu)))}
    for name, e, v, b in (("w_gate", e_dg, dg, x), ("w_up", e_du, du, x)):
        r = v.t() @ b
        out[name] = (r, bound(r, sq(e.t(), b), sq(v.t(), b)))
    r = dy.t() @ h
    out["w_down"] = (r, bound(r, sq(dy.t(), e_h), sq(dy.t(), h)))
    return out


def check(name, got, ref):
    want, tol = ref
    err = (got.double() - want).abs()
    bad = ~(err <= tol)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst {float((err / tol).max()):.2f} of it"


def run(P, T, D, F, ld, seed=0, **kw):
    x, wg, wu, wd, dy = make(T, D, F, ld, seed, **kw)
    ffn = P.Ffn(wg, wu, wd, d_ff=F)
    ws = P.alloc_workspace(P.camera_ffn_workspace_bytes(ffn, T, backward=True), DEV)
    ws.fill_(255)                                     # whatever a workspace held before
    saved = P.alloc_workspace(P.camera_ffn_saved_bytes(ffn, T), DEV).fill_(255)
    y = P.camera_ffn_forward(ffn, x, saved=saved, workspace=ws)
    assert P.camera_read_status(ws) == 0
    y2 = P.camera_ffn_forward(ffn, x)                 # nothing kept: the same output
    assert torch.equal(y, y2)
    kept = saved.clone()
    dwd = torch.full((D, ld), 7.0, dtype=torch.bfloat16, device=DEV)
    grads = P.camera_ffn_backward(ffn, x, dy, saved, workspace=ws, out={"w_down": dwd})
    assert P.camera_read_status(ws) == 0 and torch.equal(saved, kept) and grads["w_down"] is dwd
    assert (dwd[:, F:] == 7.0).all()                  # columns the block does not have are left alone
    ref = reference(x, wg, wu, wd, dy, F)
    check("y", y, ref["y"])
    for name in ("x", "w_gate", "w_up"):
        check(name, grads[name], ref[name])
    check("w_down", dwd[:, :F], ref["w_down"])
    return ffn, x, dy, saved, ws, y, grads


@pytest.mark.parametrize("T,D,F,ld", [
    (1, 8, 1, 8), (2, 16, 3, 8), (7, 64, 64, 64), (31, 72, 65, 72), (64, 128, 100, 136), (129, 200, 257, 264),
    (255, 256, 512, 512), (256, 264, 511, 512), (257, 520, 513, 520), (300, 1000, 777, 784), (513, 640, 1025, 1088),
    (1, 2048, 1408, 1408), (3, 3584, 2560, 2560), (16, 1032, 999, 1000), (17, 520, 640, 640), (33, 2048, 845, 848),
    (100, 1024, 2304, 2304), (1001, 2048, 845, 848), (2500, 512, 2049, 2056)])
def test_sizes_forward_and_backward(P, T, D, F, ld):
    run(P, T, D, F, ld, seed=T + F, w_scale=D ** -0.5)


@pytest.mark.parametrize("T", [1, 4, 8, 9, 24, 32, 48, 64, 65, 96, 128, 200])
def test_every_number_of_tokens_a_decoder_calls_with(P, T):
    D, F, ld = 1536, 1130, 1136
    x, wg, wu, wd, dy = make(T, D, F, ld, 3, w_scale=D ** -0.5)
    y = P.camera_ffn_forward(P.Ffn(wg, wu, wd, d_ff=F), x)
    check("y", y, reference(x, wg, wu, wd, dy, F)["y"])


def test_large_gates_saturate_cleanly(P):
    """Gates of either sign up to a few hundred: SiLU is g or 0 there, its derivative 1 or 0, and nothing overflows."""
    run(P, 65, 256, 192, 192, seed=1, x_scale=8.0, w_scale=2.0)


def test_results_repeat_bit_for_bit_and_parts_can_be_asked_for(P):
    ffn, x, dy, saved, ws, y, grads = run(P, 700, 512, 640, 640, w_scale=0.04)
    assert torch.equal(P.camera_ffn_forward(ffn, x, saved=saved, workspace=ws), y)
    again = P.camera_ffn_backward(ffn, x, dy, saved)
    for name, t in grads.items():
        assert torch.equal(again[name], t), name
    only_x = P.camera_ffn_backward(ffn, x, dy, saved, want_weights=False, workspace=ws)
    only_w = P.camera_ffn_backward(ffn, x, dy, saved, want_x=False, workspace=ws)
    assert set(only_x) == {"x"} and torch.equal(only_x["x"], grads["x"])
    assert set(only_w) == {"w_gate", "w_up", "w_down"} and torch.equal(only_w["w_gate"], grads["w_gate"])
    # on another stream than the tensors' own
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y2 = P.camera_ffn_forward(ffn, x, stream=side)
    side.synchronize()
    assert torch.equal(y2, y)


def test_no_tokens(P):
    x, wg, wu, wd, dy = make(4, 64, 40, 48)
    ffn = P.Ffn(wg, wu, wd, d_ff=40)
    saved = P.alloc_workspace(P.camera_ffn_saved_bytes(ffn, 0), DEV)
    assert P.camera_ffn_forward(ffn, x[:0], saved=saved).shape == (0, 64)
    dwd = torch.full((64, 48), 7.0, dtype=torch.bfloat16, device=DEV)
    grads = P.camera_ffn_backward(ffn, x[:0], dy[:0], saved, out={"w_down": dwd})
    assert grads["x"].shape == (0, 64) and not grads["w_gate"].any() and not grads["w_up"].any()
    assert not dwd[:, :40].any() and (dwd[:, 40:] == 7.0).all()


def test_a_nan_or_infinity_stays_in_its_token(P):
    T, D, F = 300, 256, 320
    x, wg, wu, wd, dy = make(T, D, F, F, 5)
    ffn = P.Ffn(wg, wu, wd)
    clean = P.camera_ffn_forward(ffn, x)
    x[17, 3] = float("nan")
    x[200, 5] = float("inf")
    y = P.camera_ffn_forward(ffn, x)
    keep = torch.ones(T, dtype=torch.bool, device=DEV)
    keep[17] = keep[200] = False
    assert torch.isnan(y[17]).all() and not torch.isfinite(y[200]).any()
    assert torch.equal(y[keep], clean[keep])
    few = P.camera_ffn_forward(ffn, x[16:20].contiguous())
    assert torch.isnan(few[1]).all() and torch.isfinite(few[[0, 2, 3]]).all()


def test_gradient_against_differences(P):
    """Directional derivatives of L = <dy, y> in float64 along a random direction of each input: the central difference
    (step 1e-4, error of order 1e-8) against the kernel's gradient, within the sum of the elements' bounds."""
    T, D, F = 40, 64, 48
    ffn, x, dy, saved, ws, y, grads = run(P, T, D, F, F, seed=2, w_scale=0.125)
    _, wg, wu, wd, _ = make(T, D, F, F, 2, w_scale=0.125)
    ref = reference(x, wg, wu, wd, dy, F)
    leaves = {"x": x, "w_gate": wg, "w_up": wu, "w_down": wd}

    def loss(v):
        g, u = v["x"] @ v["w_gate"].t(), v["x"] @ v["w_up"].t()
        return float((dy.double() * ((g * torch.sigmoid(g) * u) @ v["w_down"].t())).sum())

    base = {k: t.double() for k, t in leaves.items()}
    gen = torch.Generator(device=DEV).manual_seed(4)
    for name in leaves:
        d = torch.randn(base[name].shape, device=DEV, generator=gen, dtype=torch.float64)
        up, down = dict(base), dict(base)
        up[name], down[name] = base[name] + 1e-4 * d, base[name] - 1e-4 * d
        want = (loss(up) - loss(down)) / 2e-4
        got = float((grads[name].double() * d).sum())
        tol = float((ref[name][1] * d.abs()).sum()) + 1e-5
        assert abs(got - want) <= tol, (name, got, want, tol)


def test_a_wait_that_runs_out_is_reported(P):
    """The status word of a workspace is written by the call: a probe's timeout recorded in it does not survive."""
    x, wg, wu, wd, _ = make(400, 256, 320, 320)
    ffn = P.Ffn(wg, wu, wd)
    ws = P.alloc_workspace(P.camera_ffn_workspace_bytes(ffn, 400), DEV)
    P.camera_wait_probe(ws, 1_000_000)
    assert P.camera_read_status(ws) == -6
    P.camera_ffn_forward(ffn, x, workspace=ws)
    assert P.camera_read_status(ws) == 0
    P.camera_wait_probe(ws, 1_000_000)
    P.camera_ffn_forward(ffn, x[:1], workspace=ws)
    assert P.camera_read_status(ws) == 0
