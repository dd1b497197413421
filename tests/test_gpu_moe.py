"""Tokens sorted by expert and back, with the gradients of both, against plain forms on the same stored values.

Dispatch moves rows: exact.  combine adds k products in fp32: at most (k + 2) roundings of u = 2^-24 of the sum of magnitudes,
then one to the dtype (half a step).  combine_backward's rows are one product, rounded to fp32 and to the dtype; its weights a
sum of d products: at most d + 8 roundings of u of the sum of magnitudes.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def sort_ref(idx, experts):
    """rows, offsets and the pairs in sorted order, by Python's stable sort."""
    flat = idx.cpu().reshape(-1).tolist()
    pairs = sorted((p for p, e in enumerate(flat) if 0 <= e < experts), key=lambda p: flat[p])
    rows = [-1] * len(flat)
    for r, p in enumerate(pairs):
        rows[p] = r
    offsets = [sum(1 for e in flat if 0 <= e < x) for x in range(experts + 1)]
    return torch.tensor(rows, dtype=torch.int32).view(idx.shape), torch.tensor(offsets, dtype=torch.int32), pairs


def routing(g, tokens, k, experts, dropped=0.0, skew=False):
    idx = torch.randint(0, experts, (tokens, k), device=DEV, generator=g, dtype=torch.int32)
    if skew:
        idx = torch.where(torch.rand((tokens, k), device=DEV, generator=g) < 0.9, 0, idx)
    if dropped:
        out = torch.rand((tokens, k), device=DEV, generator=g) < dropped
        idx = torch.where(out, torch.randint(-5, 0, (tokens, k), device=DEV, generator=g, dtype=torch.int32), idx)
        idx[-1, -1] = experts                             # the first index beyond the last expert
        if tokens > 3:
            idx[2] = 2 ** 31 - 1                          # a token without any
    return idx


def matrix(g, rows, d, dtype, pad=0, first=0):
    buf = torch.zeros(rows * (d + pad) + first + 16, dtype=dtype, device=DEV)
    m = buf[first:first + rows * (d + pad)].view(rows, d + pad)[:, :d]
    m.copy_(torch.randn(rows, d, device=DEV, generator=g))
    return m


def close(got, want, tol, dtype):
    err = (got.double() - want).abs()
    tol = tol + torch.finfo(dtype).eps / 2 * (want.abs() + tol) + 1e-38
    assert (err <= tol).all(), f"worst {float((err / tol).max()):.2f} of the bound"


def gathered(rows, n, ys):
    """[T, k, d] rows of ys in float64, zeros where a pair has none."""
    ok = (rows >= 0) & (rows < n)
    return torch.where(ok[:, :, None], ys.double()[rows.clamp(0, max(n - 1, 0)).long()], 0.0), ok


SIZES = [(1, 1, 1, 8), (1, 16, 64, 3584), (2, 3, 5, 7), (33, 2, 8, 64), (64, 8, 64, 1024), (65, 6, 64, 1001), (200, 4, 1024, 72),
         (300, 16, 200, 96), (777, 6, 61, 520), (1025, 1, 3, 256), (2500, 8, 64, 136), (5000, 4, 129, 40), (3000, 8, 300, 24),
         (2049, 8, 1024, 16), (20000, 2, 256, 8)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tokens,k,experts,d", SIZES)
def test_dispatch(P, tokens, k, experts, d, dtype):
    g = torch.Generator(device=DEV).manual_seed(tokens + k)
    for dropped, skew, pad, first in ((0.0, False, 0, 0), (0.2, True, 8, 8), (0.05, False, 1, 3)):
        idx = routing(g, tokens, k, experts, dropped, skew)
        x = matrix(g, tokens, d, dtype, pad, first)
        out = matrix(g, tokens * k + 2, d, dtype, pad, first)
        before = out.clone()
        ws = P.alloc_workspace(P.camera_moe_dispatch_workspace_bytes(tokens, k, experts), DEV).fill_(255)
        r = P.camera_moe_dispatch(x, idx, experts, out=out, workspace=ws)
        rows, offsets, pairs = sort_ref(idx, experts)
        assert torch.equal(r["rows"].cpu(), rows) and torch.equal(r["offsets"].cpu(), offsets) and r["x"] is out
        n = len(pairs)
        assert torch.equal(out[:n], x[torch.tensor(pairs, dtype=torch.long, device=DEV) // k])
        assert torch.equal(out[n:], before[n:])                 # rows behind the last pair are left alone
    r2 = P.camera_moe_dispatch(x, idx, experts)
    assert torch.equal(r2["x"][:n], out[:n]) and torch.equal(r2["rows"], r["rows"])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tokens,k,experts,d", SIZES)
def test_combine_and_gradients(P, tokens, k, experts, d, dtype):
    g = torch.Generator(device=DEV).manual_seed(tokens * k)
    for dropped, weights, pad, first in ((0.0, True, 0, 0), (0.2, True, 8, 8), (0.1, False, 1, 3)):
        rows = sort_ref(routing(g, tokens, k, experts, dropped), experts)[0].to(DEV)
        n = tokens * k
        ys = matrix(g, n, d, dtype, pad, first)
        w = torch.rand((tokens, k), device=DEV, generator=g) - 0.3 if weights else None
        add = matrix(g, tokens, d, dtype, pad, first) if weights else None
        got, ok = gathered(rows, n, ys)
        wd = ok.double() if w is None else w.double() * ok
        terms = got * wd[:, :, None]
        want, size = terms.sum(1), terms.abs().sum(1)
        if add is not None:
            want, size = want + add.double(), size + add.double().abs()
        y = P.camera_moe_combine(ys, rows, w, add=add)
        close(y, want, (k + 2) * U * size, dtype)
        if add is not None:
            room = add.clone()
            assert P.camera_moe_combine(ys, rows, w, add=room, out=room) is room and torch.equal(room, y)
        else:
            assert torch.equal(P.camera_moe_dispatch_backward(ys, rows), y)
        dy = matrix(g, tokens, d, dtype, pad, first)
        out = matrix(g, n, d, dtype, pad, first)
        before = out.clone()
        r = P.camera_moe_combine_backward(dy, ys, rows, w, out=out)
        named = torch.zeros(n, dtype=torch.bool, device=DEV)
        named[rows[ok].long()] = True
        assert torch.equal(out[~named], before[~named])
        full = wd[:, :, None] * dy.double()[:, None, :]
        close(out[rows[ok].long()], full[ok], U * full[ok].abs(), dtype)
        prod = got * dy.double()[:, None, :]
        close(r["weights"], prod.sum(2), (d + 8) * U * prod.abs().sum(2), F32)
        assert not r["weights"][~ok].any()
        only = P.camera_moe_combine_backward(dy, ys, rows, w, want_y=False)
        assert set(only) == {"weights"} and torch.equal(only["weights"], r["weights"])
        room = ys.clone()
        P.camera_moe_combine_backward(dy, room, rows, w, out=room)
        assert torch.equal(room[named], out[named]) and torch.equal(room[~named], ys[~named])
        alone = P.camera_moe_combine_backward(dy, ys, rows, w, want_weights=False)
        assert set(alone) == {"y"} and torch.equal(alone["y"][named], out[named])


def test_rows_outside_the_matrix_add_nothing(P):
    ys = torch.randn(10, 64, device=DEV)
    rows = torch.tensor([[0, 10], [9, 2 ** 31 - 1], [-7, 3]], dtype=torch.int32, device=DEV)
    y = P.camera_moe_combine(ys, rows)
    assert torch.equal(y, ys[[0, 9, 3]])
    r = P.camera_moe_combine_backward(torch.ones(3, 64, device=DEV), ys, rows, out=torch.zeros(10, 64, device=DEV))
    assert (r["y"][[0, 9, 3]] == 1).all() and float(r["y"].sum()) == 3 * 64
    assert not r["weights"][[0, 1, 2], [1, 1, 0]].any()
    empty = torch.zeros(0, 64, device=DEV)
    assert not P.camera_moe_combine(empty, rows).any()
    assert not P.camera_moe_combine_backward(y, empty, rows)["weights"].any()


def test_no_tokens_and_no_pairs(P):
    x = torch.zeros(0, 32, dtype=BF, device=DEV)
    r = P.camera_moe_dispatch(x, torch.zeros(0, 4, dtype=torch.int32, device=DEV), 6)
    assert r["x"].shape == (0, 32) and r["offsets"].tolist() == [0] * 7
    assert P.camera_moe_combine(r["x"], r["rows"]).shape == (0, 32)
    assert P.camera_moe_combine_backward(x, r["x"], r["rows"])["weights"].shape == (0, 4)
    none = torch.full((5, 4), -1, dtype=torch.int32, device=DEV)
    out = torch.full((20, 32), 7.0, dtype=BF, device=DEV)
    r = P.camera_moe_dispatch(torch.ones(5, 32, dtype=BF, device=DEV), none, 6, out=out)
    assert (out == 7.0).all() and torch.equal(r["rows"], none) and not r["offsets"].any()
    assert torch.equal(P.camera_moe_combine(out, r["rows"], add=out[:5]), out[:5])


def test_there_and_back_is_the_sum_of_the_weights(P):
    """Experts that change nothing: y[t] = x[t] times the sum of its weights, and x's gradient is dy times that sum."""
    g = torch.Generator(device=DEV).manual_seed(1)
    T, k, d = 513, 4, 256
    idx = torch.rand((T, 16), device=DEV, generator=g).topk(k, 1).indices.int()
    w = torch.softmax(torch.randn((T, k), device=DEV, generator=g), 1)
    x, dy = torch.randn((T, d), device=DEV, generator=g), torch.randn((T, d), device=DEV, generator=g)
    s = P.camera_moe_dispatch(x, idx, 16)
    y = P.camera_moe_combine(s["x"], s["rows"], w)
    back = P.camera_moe_combine_backward(dy, s["x"], s["rows"], w)
    dx = P.camera_moe_dispatch_backward(back["y"], s["rows"])
    assert torch.allclose(y, x, rtol=1e-6, atol=1e-6) and torch.allclose(dx, dy, rtol=1e-6, atol=1e-6)
    dots = (x.double() * dy.double()).sum(1, keepdim=True)
    assert torch.allclose(back["weights"].double(), dots.expand(T, k), atol=1e-4)


def test_repeats_bit_for_bit_on_another_stream_and_in_a_graph(P):
    g = torch.Generator(device=DEV).manual_seed(2)
    T, k, E, d = 4096, 8, 64, 256
    idx, x = routing(g, T, k, E, 0.1), torch.randn((T, d), device=DEV, generator=g).bfloat16()
    w, dy = torch.rand((T, k), device=DEV, generator=g), torch.randn((T, d), device=DEV, generator=g).bfloat16()
    ws = P.alloc_workspace(P.camera_moe_dispatch_workspace_bytes(T, k, E), DEV)
    out, back = torch.zeros((T * k, d), dtype=BF, device=DEV), torch.zeros((T * k, d), dtype=BF, device=DEV)

    def all_of_it():
        s = P.camera_moe_dispatch(x, idx, E, out=out, workspace=ws)
        y = P.camera_moe_combine(s["x"], s["rows"], w, add=x)
        r = P.camera_moe_combine_backward(dy, s["x"], s["rows"], w, out=back)
        return [s["rows"], s["offsets"], y, r["weights"], P.camera_moe_dispatch_backward(r["y"], s["rows"], add=dy), out, back]

    first = [t.clone() for t in all_of_it()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = all_of_it()
    side.synchronize()
    for a, b in zip(first, again):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = all_of_it()
    idx.copy_(routing(g, T, k, E, 0.3))
    x.copy_(torch.randn((T, d), device=DEV, generator=g))
    out.zero_(), back.zero_()
    graph.replay()
    torch.cuda.synchronize()
    held = [t.clone() for t in held]
    out.zero_(), back.zero_()
    for a, b in zip(held, all_of_it()):
        assert torch.equal(a, b)
