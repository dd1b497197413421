"""Orthogonalised updates of matrices of low rank, as an expert's gradient is that few tokens reached, against float64.

What a rounding of X puts where the matrix has nothing grows by the polynomial's slope at 0 in every step left, so it decides what
these matrices are off by.  Tolerance, derived before the first run: `modelled` does in float64 the roundings that X, A and B
are held with (X as two fp16 numbers of which the products take the first; the diagonals of A and B as if kept), and the bound is
twice its error (Frobenius norm), plus 2^-8 / sqrt(3) of the result for the rounding to bf16, plus the fp32 sums: of k products, 16 at a
time, k / 16 roundings of 2^-23 at most, sqrt(k / 16) 2^-23 <= 2^-20 in the root mean square for k <= 1024, grown by the product of
the steps' slopes.
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
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(m * 2048) / 2048, e)


def kept_diagonal(x):
    return half(x) + torch.diag_embed(torch.diagonal(x) - half(torch.diagonal(x)))


def modelled(u, coefficients, rounded, eps=1e-7):
    x = u.double()
    flip = x.shape[0] > x.shape[1]
    x = x.t() if flip else x
    x = x / (x.norm() + eps)
    low = torch.zeros_like(x)
    if rounded:
        x, low = half(x), half(x - half(x))
    for i, (a, b, c) in enumerate(coefficients):
        gram = x @ x.t()
        gram = kept_diagonal(gram) if rounded else gram
        mat = b * gram + c * (gram @ gram)
        mat.diagonal().add_(a)
        mat = kept_diagonal(mat) if rounded else mat
        x = mat @ x
        if rounded:
            growth = 1.0
            for later in coefficients[i + 1:]:
                growth *= max(1.0, abs(later[0]))
            x = x + (a + (torch.diagonal(mat) - a)[:, None] / (1 + (growth / 8) ** 2)) * low
            if i + 1 < len(coefficients):
                x, low = half(x), half(x - half(x))
    return x.t() if flip else x


def check(got, u, coefficients):
    want = modelled(u, coefficients, False)
    off = float((modelled(u, coefficients, True) - want).norm())
    slopes = 1.0
    for a, _, _ in coefficients:
        slopes *= max(1.0, abs(a))
    bound = 2 * off + (2.0 ** -8 / 3 ** 0.5 + 2.0 ** -20 * slopes) * float(want.norm()) + 1e-30
    err = float((got.double() - want).norm())
    assert err <= bound, (err / float(want.norm()), bound / float(want.norm()))


def of_rank(g, r, c, rank, dtype):
    """A gradient made from `rank` tokens."""
    left = torch.randn((rank, r), device=DEV, generator=g) * torch.exp(torch.randn(r, device=DEV, generator=g) * 0.5)
    right = torch.randn((rank, c), device=DEV, generator=g) * torch.linspace(0, -2, c, device=DEV).exp()
    return (left.t() @ right * (1e-3 / rank)).to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("r,c", [(64, 300), (300, 64), (512, 1024), (257, 257), (1000, 513), (40, 2000)])
def test_gradients_of_few_tokens(P, r, c, dtype):
    g = torch.Generator(device=DEV).manual_seed(r + c)
    us = [of_rank(g, r, c, t, dtype) for t in (1, 2, 8, 64, min(r, c) // 2 + 1)]
    for u, o in zip(us, P.camera_orthogonalize(us)):
        check(o, u, [P.NEWTON_SCHULZ] * 5)


def test_a_gradient_of_one_token_is_its_direction(P):
    """Rank one: the result is the matrix over its norm, times what the polynomial makes of 1."""
    g = torch.Generator(device=DEV).manual_seed(1)
    u = of_rank(g, 512, 1024, 1, F32)
    s = 1.0
    for _ in range(5):
        a, b, c = P.NEWTON_SCHULZ
        s = s * (a + b * s ** 2 + c * s ** 4)
    want = s * u.double() / u.double().norm()
    err = float((P.camera_orthogonalize([u])[0].double() - want).norm() / want.norm())
    assert err < 5e-3, err


def test_rows_and_columns_of_zeros(P):
    """Units that no token moved: their rows and columns stay near zero beside the others'."""
    g = torch.Generator(device=DEV).manual_seed(2)
    u = torch.randn(300, 700, device=DEV, generator=g)
    u[50:250] = 0
    u[:, 100:600] = 0
    o = P.camera_orthogonalize([u])[0]
    check(o, u, [P.NEWTON_SCHULZ] * 5)
    assert not o[50:250].any() and not o[:, 100:600].any()


@pytest.mark.parametrize("name", ["cubic", "mixed"])
def test_other_polynomials(P, name):
    g = torch.Generator(device=DEV).manual_seed(3)
    coefficients = {"cubic": [(1.5, -0.5, 0.0)] * 12, "mixed": [(3.4445, -4.775, 2.0315), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)]}[name]
    for rank in (1, 8, 100):
        u = of_rank(g, 150, 400, rank, F32)
        check(P.camera_orthogonalize([u], coefficients=coefficients)[0], u, coefficients)
        small = u * 1e-9
        check(P.camera_orthogonalize([small], coefficients=coefficients, eps=0.0)[0], u, coefficients)


@pytest.mark.parametrize("shapes,dtype", [
    ([(3329, 3555)], F32), ([(3600, 3333)], BF), ([(2048, 8192)], F32), ([(2810, 2603)], BF),
    ([(1408 - 37 * i, 2048) if i % 3 else (2048, 1408 - 37 * i) for i in range(16)], F32)], ids=lambda v: str(v[0]) if isinstance(v, list) else "")
def test_gradients_of_few_tokens_in_wide_tiles(P, shapes, dtype):
    """Tiles of 256 and of twice 256 columns.  Sums of k products: sqrt(k / 16) 2^-23, as above, grown by the slopes."""
    g = torch.Generator(device=DEV).manual_seed(len(shapes))
    coefficients = [P.NEWTON_SCHULZ] * 5
    us = [of_rank(g, r, c, 1 + 7 * (i % 5), dtype) for i, (r, c) in enumerate(shapes)]
    for u, o in zip(us, P.camera_orthogonalize(us)):
        want = modelled(u, coefficients, False)
        off = float((modelled(u, coefficients, True) - want).norm())
        sums = (min(u.shape) / 16) ** 0.5 * 2.0 ** -23 * P.NEWTON_SCHULZ[0] ** 5
        bound = 2 * off + (2.0 ** -8 / 3 ** 0.5 + sums) * float(want.norm())
        assert float((o.double() - want).norm()) <= bound, (float((o.double() - want).norm()), bound)
