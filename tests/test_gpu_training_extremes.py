"""The operators around a layer's experts where sizes pass 2^31, where threads and streams call at once, and where a caller's own CUDA
error state must stay as it was."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF = torch.bfloat16


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def test_norm_of_more_than_2_31_elements(P):
    rows, d = 262145, 8208                                  # 2.15e9 elements, 4.3 GB a matrix
    x = torch.empty(rows, d, dtype=BF, device=DEV)
    x[:1000].normal_(), x[-1000:].normal_()
    x[1000:-1000] = 0.5
    out = P.camera_norm_forward(x, rms=True)
    for part in (slice(0, 1000), slice(rows - 1000, rows)):
        small = P.camera_norm_forward(x[part], rms=True)    # fewer rows, another kernel shape: sums in another order
        assert torch.allclose(out["rstd"][part], small["rstd"], rtol=1e-5)
        assert torch.allclose(out["y"][part].float(), small["y"].float(), rtol=2 ** -6, atol=1e-6)
    y = out["y"]
    del out["y"]
    # dx over x's own room; rows of equal elements have no gradient along them
    dy = y.fill_(1.0)
    grads = P.camera_norm_backward(dy, x, out["rstd"], out=x)
    h = grads["weight"]
    assert torch.isfinite(h).all() and float(x[1000:-1000].float().abs().max()) < 1e-2
    del x, y, dy, grads, out
    torch.cuda.empty_cache()


def test_sorted_rows_of_more_than_2_31_elements(P):
    T, k, E, d = 33000, 8, 64, 8192                         # 264000 rows, 2.16e9 elements
    g = torch.Generator(device=DEV).manual_seed(0)
    idx = torch.randint(0, E, (T, k), device=DEV, generator=g, dtype=torch.int32)
    x = torch.randn(T, d, device=DEV, generator=g).bfloat16()
    s = P.camera_moe_dispatch(x, idx, E)
    rows = s["rows"].long()
    assert int(s["offsets"][-1]) == T * k
    pick = torch.cat([torch.arange(500), torch.arange(T - 500, T)]).to(DEV)
    assert torch.equal(s["x"][rows[pick].reshape(-1)], x[pick].repeat_interleave(k, 0))
    last = torch.full_like(rows, -1).scatter_(1, rows.argmax(1, keepdim=True), rows.max(1, keepdim=True).values).int()
    y = P.camera_moe_combine(s["x"], last)                  # of each token the row that lies furthest back
    assert torch.equal(y, x)
    back = P.camera_moe_combine_backward(x, s["x"], s["rows"], want_weights=True, out=s["x"])
    assert torch.equal(back["y"][rows[pick].reshape(-1)], x[pick].repeat_interleave(k, 0))
    want = x[pick].double().pow(2).sum(1, keepdim=True).expand(-1, k)
    assert torch.allclose(back["weights"][pick].double(), want, rtol=1e-4)
    del s, x, y, back
    torch.cuda.empty_cache()


def test_threads_with_streams_of_their_own(P):
    """Calls of several host threads at once, each with its workspaces: the results of one after the other."""
    def work(seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        x = torch.randn(300 + seed, 512, device=DEV, generator=g).bfloat16()
        idx = torch.randint(0, 16, (300 + seed, 4), device=DEV, generator=g, dtype=torch.int32)
        u = [torch.randn(100 + 20 * seed, 300, device=DEV, generator=g), torch.randn(130, 90, device=DEV, generator=g)]
        f = P.camera_norm_forward(x, rms=False)
        b = P.camera_norm_backward(x, x, f["rstd"], f["mean"])
        s = P.camera_moe_dispatch(f["y"], idx, 16)
        return [f["y"], b["x"], b["weight"], s["x"], P.camera_moe_combine(s["x"], s["rows"])] + P.camera_orthogonalize(u)

    alone = [[t.clone() for t in work(i)] for i in range(4)]
    torch.cuda.synchronize()
    got, errors = [None] * 4, []

    def thread(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(5):
                    got[i] = work(i)
            stream.synchronize()
        except Exception as e:      # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=thread, args=(i,)) for i in range(4)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not errors, errors
    for a, b in zip(alone, got):
        for s, t in zip(a, b):
            assert torch.equal(s, t)


def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right(P):
    """With a limit of 1 us units that wait for others give up: the call ends, says so, and nothing is left behind."""
    g = torch.Generator(device=DEV).manual_seed(3)
    u = [torch.randn(700, 900, device=DEV, generator=g) for _ in range(3)]
    ws = P.alloc_workspace(P.camera_orthogonalize_workspace_bytes(u), DEV)
    want = P.camera_orthogonalize(u, workspace=ws)
    assert P.camera_read_status(ws) == 0
    before = P.camera_get_wait_limit_ns()
    P.camera_set_wait_limit_ns(1000)
    try:
        P.camera_orthogonalize(u, workspace=ws)
        assert P.camera_read_status(ws) == -6
    finally:
        P.camera_set_wait_limit_ns(before)
    for a, b in zip(want, P.camera_orthogonalize(u, workspace=ws)):
        assert torch.equal(a, b)
    assert P.camera_read_status(ws) == 0


def test_more_matrices_than_one_launch_takes(P):
    """Rounds of 64 matrices share the workspace one after the other; results are those of each round alone."""
    g = torch.Generator(device=DEV).manual_seed(4)
    u = [torch.randn(30 + i % 7, 50 + i, device=DEV, generator=g).bfloat16() for i in range(150)]
    all_of_them = P.camera_orthogonalize(u)
    parts = [o for a in range(0, 150, 64) for o in P.camera_orthogonalize(u[a:a + 64])]
    for a, b in zip(all_of_them, parts):
        assert torch.equal(a, b)


def test_a_refused_call_leaves_no_error_behind(P):
    x = torch.randn(8, 64, device=DEV)
    with pytest.raises(P.CameraError):
        P.camera_norm_forward(x, eps=-1.0)
    with pytest.raises(P.CameraError):
        P.camera_moe_dispatch(x, torch.zeros(8, 17, dtype=torch.int32, device=DEV), 4, workspace=P.alloc_workspace(256, DEV))
    with pytest.raises(P.CameraError):
        P.camera_orthogonalize([x], coefficients=(5000.0, 0.0, 0.0))
    with pytest.raises(P.CameraError):
        P.camera_orthogonalize([x], workspace=P.alloc_workspace(256, DEV))
    with pytest.raises(ValueError):
        P.camera_norm_forward(x.t())
    with pytest.raises(ValueError):
        P.camera_moe_combine(x, torch.zeros(8, 2, dtype=torch.int64, device=DEV))
    torch.cuda.synchronize()
    assert torch.isfinite(P.camera_norm_forward(x)["y"]).all()


def test_almost_2_31_tokens(P):
    """As many tokens as a call takes, one column: token numbers and counts of CTAs near the end of 31 bits."""
    T = 2 ** 31 - 5
    idx = torch.zeros(T, 1, dtype=torch.int32, device=DEV)
    idx[-3:] = 1
    idx[5] = -1
    x = torch.empty(T, 1, dtype=BF, device=DEV).random_(0, 200)
    s = P.camera_moe_dispatch(x, idx, 2)
    assert s["offsets"].tolist() == [0, T - 4, T - 1]
    rows, step = s["rows"].view(-1), 2 ** 28
    for a in range(0, T, step):
        want = torch.arange(a, min(a + step, T), device=DEV)
        want = torch.where(want == 5, -1, want - (want > 5).long())
        assert torch.equal(rows[a:a + step].long(), want)
        del want
    assert torch.equal(s["x"][:5], x[:5]) and torch.equal(s["x"][5:-1], x[6:])
    del idx
    y = P.camera_moe_combine(s["x"][:-1], s["rows"])
    assert y[5, 0] == 0 and torch.equal(y[:5], x[:5]) and torch.equal(y[6:], x[6:])
    s["x"][-1] = 3.0
    back = P.camera_moe_combine_backward(y, s["x"], s["rows"], want_weights=False)["y"]
    assert torch.equal(back[:5], x[:5]) and torch.equal(back[5:-1], x[6:])
    del x, s, y, back, rows
    torch.cuda.empty_cache()
