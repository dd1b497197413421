"""Orthogonalised updates against float64.

Tolerance, derived before the first run.  Apart from fp32 sums the kernels differ from the definition by roundings: X, A and B
to fp16 (the diagonals of A and B as if kept) and the result to bf16.  `modelled` does the same roundings in float64; what it is
off by is how far these roundings move this matrix's result.  The kernel's roundings fall elsewhere in detail, so its error
before the last rounding is of that size but not that value: the bound is twice it (Frobenius norm), plus 1e-5 for the sums, plus
2^-8 / sqrt(3) of the result for its rounding (uniform within half a step, 2^-8).  An element's bound is 2^-8 of its value plus
four times the largest element error of the model.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def half(x):
    """Rounded to the 11 bits of fp16, without its range."""
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(m * 2048) / 2048, e)


def without_diagonal(x):
    return half(x) + torch.diag_embed(torch.diagonal(x) - half(torch.diagonal(x)))


def definition(u, coefficients, eps=1e-7, rounded=False):
    x = u.double()
    flip = x.shape[0] > x.shape[1]
    x = x.t() if flip else x
    x = x / (x.norm() + eps)
    if rounded:
        x = half(x)
    eye = torch.eye(x.shape[0], device=DEV, dtype=torch.float64)
    for i, (a, b, c) in enumerate(coefficients):
        gram = x @ x.t()
        if rounded:
            gram = without_diagonal(gram)
        mat = a * eye + b * gram + c * (gram @ gram)
        if rounded:
            mat = without_diagonal(mat)
        x = mat @ x
        if rounded and i + 1 < len(coefficients):
            x = half(x)
    return x.t() if flip else x


def check(got, u, coefficients, eps=1e-7):
    want, model = definition(u, coefficients, eps), definition(u, coefficients, eps, True)
    assert got.shape == u.shape and got.dtype is BF
    off = (model - want)
    err = got.double() - want
    bound = 2 * float(off.norm()) + (1e-5 + 2.0 ** -8 / 3 ** 0.5) * float(want.norm()) + 1e-30
    assert float(err.norm()) <= bound, (float(err.norm()), bound)
    each = 2.0 ** -8 * want.abs() + 4 * float(off.abs().max()) + 1e-4 * float(want.abs().max()) + 1e-30
    assert (err.abs() <= each).all(), float((err.abs() / each).max())


def update(g, r, c, dtype=BF, pad=0, first=0, kind="gauss"):
    u = torch.randn(r, c, device=DEV, generator=g)
    if kind == "decay":
        u = u * torch.linspace(0, -3, c, device=DEV).exp() * torch.exp(torch.randn(r, 1, device=DEV, generator=g) * 0.5)
    if kind == "alike":
        q = torch.linalg.qr(torch.randn(max(r, c), min(r, c), device=DEV, generator=g))[0]
        u = q if r >= c else q.t()
    buf = torch.zeros(r * (c + pad) + first + 8, dtype=dtype, device=DEV)
    m = buf[first:first + r * (c + pad)].view(r, c + pad)[:, :c]
    m.copy_(u * 1e-3)
    return m


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("r,c", [(1, 1), (1, 300), (300, 1), (2, 2), (8, 40), (33, 1000), (64, 64), (65, 63), (100, 300), (300, 100), (128, 512), (255, 257),
                                 (256, 256), (257, 513), (512, 300), (513, 520), (700, 1100), (1030, 900), (845, 2048)])
def test_sizes(P, r, c, dtype):
    g = torch.Generator(device=DEV).manual_seed(r * c)
    for kind in ("gauss", "decay", "alike"):
        u = update(g, r, c, dtype, kind=kind)
        ws = P.alloc_workspace(P.camera_orthogonalize_workspace_bytes([u]), DEV).fill_(255)
        got = P.camera_orthogonalize([u], workspace=ws)[0]
        assert P.camera_read_status(ws) == 0
        check(got, u, [P.NEWTON_SCHULZ] * 5)


def test_many_shapes_in_one_call(P):
    g = torch.Generator(device=DEV).manual_seed(5)
    shapes = [(300, 700), (700, 300), (1, 5), (64, 64), (513, 257), (0, 10), (40, 2000), (257, 900), (12, 0)] + [(96 + 7 * i, 160) for i in range(70)]
    us = [update(g, r, c, pad=i % 3, first=i % 2) for i, (r, c) in enumerate(shapes)]
    outs = P.camera_orthogonalize(us)
    for u, o in zip(us, outs):
        assert o.shape == u.shape
        if u.numel():
            check(o, u, [P.NEWTON_SCHULZ] * 5)


def test_strided_results_and_in_place(P):
    g = torch.Generator(device=DEV).manual_seed(6)
    for r, c in ((200, 333), (333, 200), (130, 256), (256, 130)):
        for pad, first in ((0, 0), (3, 1), (8, 8), (2, 2)):
            u = update(g, r, c, BF, pad, first)
            want = P.camera_orthogonalize([u.contiguous()])[0]
            buf = torch.full((r * (c + pad) + first + 8,), 7.0, dtype=BF, device=DEV)
            o = buf[first:first + r * (c + pad)].view(r, c + pad)[:, :c]
            assert torch.equal(P.camera_orthogonalize([u], out=[o])[0], want)
            assert (buf[:first] == 7.0).all() and (buf[first + r * (c + pad):] == 7.0).all()
            if pad:
                assert (buf[first:first + r * (c + pad)].view(r, c + pad)[:, c:] == 7.0).all()
            P.camera_orthogonalize([u], out=[u])
            assert torch.equal(u, want)


def test_a_tensor_of_matrices_and_other_polynomials(P):
    g = torch.Generator(device=DEV).manual_seed(7)
    u = torch.randn(3, 150, 400, device=DEV, generator=g)
    o = P.camera_orthogonalize(u)
    assert o.shape == u.shape
    for i in range(3):
        check(o[i], u[i], [P.NEWTON_SCHULZ] * 5)
    # the cubic iteration towards 1, and a list with other coefficients for each step
    cubic = [(1.5, -0.5, 0.0)] * 12
    check(P.camera_orthogonalize([u[0]], coefficients=cubic)[0], u[0], cubic)
    mixed = [(3.4445, -4.775, 2.0315), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)]
    check(P.camera_orthogonalize([u[1]], coefficients=mixed)[0], u[1], mixed)
    check(P.camera_orthogonalize([u[2]], steps=1)[0], u[2], [P.NEWTON_SCHULZ])


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1.0, 1e12, 1e30])
def test_any_scale(P, scale):
    g = torch.Generator(device=DEV).manual_seed(8)
    u = torch.randn(70, 190, device=DEV, generator=g) * scale
    check(P.camera_orthogonalize([u], eps=0.0)[0], u, [P.NEWTON_SCHULZ] * 5, 0.0)
    check(P.camera_orthogonalize([u], eps=1e-7)[0], u, [P.NEWTON_SCHULZ] * 5, 1e-7)


def test_zeros_and_what_is_not_finite(P):
    g = torch.Generator(device=DEV).manual_seed(9)
    us = [torch.randn(90, 200, device=DEV, generator=g) for _ in range(4)]
    clean = P.camera_orthogonalize(us)
    us[1] = torch.zeros(90, 200, device=DEV)
    us[2][5, 7] = float("nan")
    us[3][80, 3] = float("inf")
    o = P.camera_orthogonalize(us)
    assert torch.equal(o[0], clean[0]) and not o[1].any() and torch.isnan(o[2]).all() and torch.isnan(o[3]).all()
    assert not P.camera_orthogonalize([us[1]], eps=0.0)[0].any()
    # a workspace that has seen NaN serves the next call
    ws = P.alloc_workspace(P.camera_orthogonalize_workspace_bytes(us), DEV)
    P.camera_orthogonalize(us, workspace=ws)
    small = [us[0][:70, :130].contiguous()]
    assert torch.equal(P.camera_orthogonalize(small, workspace=ws)[0], P.camera_orthogonalize(small)[0])


def test_nothing_to_do(P):
    assert P.camera_orthogonalize([]) == []
    ws = P.alloc_workspace(1 << 20, DEV).fill_(255)
    assert P.camera_orthogonalize([torch.zeros(0, 8, device=DEV)], workspace=ws)[0].shape == (0, 8)
    assert P.camera_read_status(ws) == 0


def test_repeats_bit_for_bit_on_another_stream_and_in_a_graph(P):
    g = torch.Generator(device=DEV).manual_seed(10)
    us = [update(g, 400, 900), update(g, 900, 400), update(g, 333, 500)]
    ws = P.alloc_workspace(P.camera_orthogonalize_workspace_bytes(us), DEV)
    first = P.camera_orthogonalize(us, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = P.camera_orthogonalize(us, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = P.camera_orthogonalize(us, workspace=ws)
    graph.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(first, again, held):
        assert torch.equal(a, b) and torch.equal(a, c)
    us[0].copy_(update(g, 400, 900))
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(held, P.camera_orthogonalize(us)):
        assert torch.equal(a, b)


def test_the_status_word_is_the_calls_own(P):
    u = [torch.randn(64, 64, device=DEV)]
    ws = P.alloc_workspace(P.camera_orthogonalize_workspace_bytes(u), DEV)
    P.camera_wait_probe(ws, 1_000_000)
    assert P.camera_read_status(ws) == -6
    P.camera_orthogonalize(u, workspace=ws)
    assert P.camera_read_status(ws) == 0
