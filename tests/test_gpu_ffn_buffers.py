"""Buffers of the feed-forward block: one workspace over calls of many sizes, and gradients that take an input's room."""
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


@pytest.mark.parametrize("D,F,most,tokens", [
    (3584, 2560, 2476, (1, 64, 65, 150, 203, 257, 511, 700, 2476)),
    (2048, 1408, 1853, (65, 100, 256, 380, 1853)),
    (1024, 9000, 700, (65, 66, 100, 129, 300, 700))])
def test_a_workspace_for_the_largest_call_serves_smaller_ones(P, D, F, most, tokens):
    """Against a call with a workspace of its own.  Sums over k are cut into at most 8 parts of fp32 sums; a different
    cut moves an fp32 sum of bf16 products by a few 2^-24 of the sum of magnitudes, so results may differ by one
    rounding to bf16 (2^-7 of the value next to a power of two) and values near 0 by 2^-20 of the typical size."""
    ffn, x, dy = make(P, most, D, F, F)
    for backward in (False, True):
        ws = P.alloc_workspace(P.camera_ffn_workspace_bytes(ffn, most, backward=backward), DEV)
        for T in tokens:
            xt, dyt = x[:T], dy[:T]
            saved = P.alloc_workspace(P.camera_ffn_saved_bytes(ffn, T), DEV) if backward else None
            got = {"y": P.camera_ffn_forward(ffn, xt, saved=saved, workspace=ws)}
            want = {"y": P.camera_ffn_forward(ffn, xt)}
            if backward:
                got.update(P.camera_ffn_backward(ffn, xt, dyt, saved, workspace=ws))
                want.update(P.camera_ffn_backward(ffn, xt, dyt, saved))
            assert P.camera_read_status(ws) == 0
            for name in want:
                a, b = got[name].double(), want[name].double()
                tol = 2.0 ** -7 * b.abs() + 2.0 ** -20 * b.abs().mean() * 16
                assert ((a - b).abs() <= tol).all(), (T, name, float(((a - b).abs() - tol).max()))


def test_the_teachers_workspace_serves_a_narrower_student(P):
    D, F, T = 512, 2048, 700
    teacher, x, dy = make(P, T, D, F, F)
    ws = P.alloc_workspace(P.camera_ffn_workspace_bytes(teacher, T, backward=True), DEV)
    for f in (1792, 1760, 1729, 1500, 1000, 77, 1):
        student = P.Ffn(teacher.w_gate, teacher.w_up, teacher.w_down, d_ff=f)
        saved = P.alloc_workspace(P.camera_ffn_saved_bytes(student, T), DEV)
        P.camera_ffn_forward(student, x, saved=saved, workspace=ws)
        P.camera_ffn_backward(student, x, dy, saved, workspace=ws)
        assert P.camera_read_status(ws) == 0


@pytest.mark.parametrize("T,D,F,ld", [(40, 64, 48, 48), (300, 520, 333, 336), (1001, 1024, 845, 848)])
def test_the_gradient_by_x_may_take_the_room_of_x_or_dy(P, T, D, F, ld):
    ffn, x, dy = make(P, T, D, F, ld)
    saved = P.alloc_workspace(P.camera_ffn_saved_bytes(ffn, T), DEV)
    P.camera_ffn_forward(ffn, x, saved=saved)
    w_down = lambda: torch.zeros(D, ld, dtype=torch.bfloat16, device=DEV)
    want = P.camera_ffn_backward(ffn, x, dy, saved, out={"w_down": w_down()})
    for over in ("x", "dy"):
        x2, dy2 = x.clone(), dy.clone()
        got = P.camera_ffn_backward(ffn, x2, dy2, saved, out={"x": x2 if over == "x" else dy2, "w_down": w_down()})
        for name in want:
            assert torch.equal(got[name], want[name]), (over, name)
