"""What a forward call keeps for its backward call: gate and up products with 24 bits in two planes, by both of the kernels
that write them (up to 64 tokens, and more), and read whole by the backward pass."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def make(P, T, D, F, ld, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(s, device=DEV, generator=g)
    w = [(r(F, D) * D ** -0.5).bfloat16(), (r(F, D) * D ** -0.5).bfloat16(), (r(D, ld) * F ** -0.5).bfloat16()]
    return P.Ffn(*w, d_ff=F), r(T, D).bfloat16(), (r(T, D) * 0.1).bfloat16()


@pytest.mark.parametrize("T", [1, 24, 64, 65, 300])
def test_the_products_kept_for_the_backward_pass_have_24_bits(P, T):
    """Both planes of `saved` (upper 16 bits of G and U by rows of 2 * pitch, then their lower 8 bits) against float64.  A
    product is an fp32 sum of D bf16 products (error below 2^-18 of the root of the sum of squares here) cut to 24 bits
    (relative error below 2^-15)."""
    D, F = 512, 333
    ffn, x, _ = make(P, T, D, F, 336)
    n = P.camera_ffn_saved_bytes(ffn, T)
    saved = P.alloc_workspace(n, DEV).zero_()
    P.camera_ffn_forward(ffn, x, saved=saved)
    pitch = (F + 63) // 64 * 64
    low_at = (4 * T * pitch + 1 + 255) // 256 * 256
    hi = saved[: 4 * T * pitch].view(torch.int16).view(T, 2, pitch)[:, :, :F].int() & 0xffff
    lo = saved[low_at: low_at + 2 * T * pitch].view(T, 2, pitch)[:, :, :F].int()
    got = ((hi << 16) | (lo << 8)).view(torch.float32).double()
    for i, w in enumerate((ffn.w_gate, ffn.w_up)):
        want = x.double() @ w.double().t()
        size = (x.double().square() @ w.double().square().t()).sqrt()
        assert ((got[:, i] - want).abs() <= 2.0 ** -15 * want.abs() + 2.0 ** -17 * size).all()


@pytest.mark.parametrize("T", [24, 64, 65, 300])
def test_the_backward_pass_reads_all_of_them(P, T):
    """Without the lower bytes G and U are cut to bf16 (errors up to 2^-8, all towards 0) and the weight gradients lose: their
    other roundings, of dG and dU to bf16 (up to 2^-9 either way) and of the result, leave an error of about 1.2 2^-9 in all
    (root mean square, relative), G and U in bf16 one that is larger by half at least.  0.8 lies between."""
    D, F = 512, 333
    ffn, x, dy = make(P, T, D, F, 336)
    saved = P.alloc_workspace(P.camera_ffn_saved_bytes(ffn, T), DEV).zero_()
    P.camera_ffn_forward(ffn, x, saved=saved)
    cut = saved.clone()
    pitch = (F + 63) // 64 * 64
    cut[(4 * T * pitch + 1 + 255) // 256 * 256:] = 0
    whole, less = P.camera_ffn_backward(ffn, x, dy, saved), P.camera_ffn_backward(ffn, x, dy, cut)
    xd, dyd, wg, wu, wd = (t.double() for t in (x, dy, ffn.w_gate, ffn.w_up, ffn.w_down[:, :F]))
    g, u, dh = xd @ wg.t(), xd @ wu.t(), dyd @ wd
    s = torch.sigmoid(g)
    want = {"w_gate": (dh * u * s * (1 + g * (1 - s))).t() @ xd, "w_up": (dh * g * s).t() @ xd}
    for name, r in want.items():
        off = [float((t[name].double() - r).norm() / r.norm()) for t in (whole, less)]
        assert off[0] < 0.8 * off[1] and off[0] < 2.0 * 2.0 ** -9, (name, off)
