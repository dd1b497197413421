"""The operators around a layer's experts as they are used together: a block x + MoE(norm(x)), forward and backward, against
float64 with the same routing; and the example runs.

Tolerance, derived before the first run.  Between the calls values are rounded to bf16 (half a step u = 2^-8, so a relative error
of at most u, u / sqrt(3) in the root mean square for errors spread evenly): the norm's output, the experts' gated product and
output, in the backward pass the gradients of the experts' outputs, of gate and up, of the experts' inputs and of the normalised
rows.  A result has passed at most 8 such roundings, each of which moves it by at most u / sqrt(3) of its size in the root mean
square times how far the part it is in is larger than the result; sums of gradients cancel by a factor of at most 4 at these
sizes (the parts added are of the size of the sum).  So relative errors (2-norm) are below 4 sqrt(8) u / sqrt(3) = 0.026.  An
expert's matrices are sums over its own tokens: the same bound.
"""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
DEV = "cuda:0"
BOUND = 4 * 8 ** 0.5 * 2.0 ** -8 / 3 ** 0.5


def rel(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("tokens,d,experts,k", [(257, 128, 5, 2), (64, 256, 8, 4), (1, 64, 4, 2)])
def test_a_block_and_its_gradients(tokens, d, experts, k):
    import paper_2508_02322_b200 as P
    from recover_layer import Block
    g = torch.Generator(device=DEV).manual_seed(tokens)
    rnd = lambda *s: torch.randn(s, device=DEV, generator=g)
    widths = [40 + 23 * e for e in range(experts)]                                # sliced experts: each another width
    mats = [((rnd(f, d) * d ** -0.5).bfloat16(), (rnd(f, d) * d ** -0.5).bfloat16(), (rnd(d, (f + 7) // 8 * 8) * f ** -0.5).bfloat16()) for f in widths]
    norm_weight, w_router = (1 + 0.1 * rnd(d)).bfloat16(), (rnd(experts, d) * d ** -0.5).bfloat16()
    block = Block(norm_weight, w_router, [P.Ffn(*m, d_ff=f) for m, f in zip(mats, widths)], k, tokens)
    x, dy = rnd(tokens, d).bfloat16(), rnd(tokens, d).bfloat16()
    y = block.forward(x)
    idx = block.kept[2]
    grads = block.backward(dy)

    leaf = lambda t: t.double().requires_grad_()
    xd, nd, rd = leaf(x), leaf(norm_weight), leaf(w_router)
    md = [[leaf(t[:, :f] if i == 2 else t) for i, t in enumerate(m)] for m, f in zip(mats, widths)]
    h = xd * (xd.pow(2).mean(1, keepdim=True) + 1e-6).rsqrt() * nd
    p = torch.softmax(h @ rd.t(), 1).gather(1, idx)
    w = p / p.sum(1, keepdim=True)
    out = xd
    for e, (wg, wu, wd) in enumerate(md):
        share = (w * (idx == e)).sum(1, keepdim=True)
        out = out + share * ((torch.nn.functional.silu(h @ wg.t()) * (h @ wu.t())) @ wd.t())
    want = torch.autograd.grad(out, [xd, nd, rd] + [t for m in md for t in m], dy.double(), allow_unused=True)
    assert rel(y, out.detach()) < BOUND
    assert rel(grads["x"], want[0]) < BOUND
    assert rel(grads["norm"], want[1]) < BOUND
    assert rel(grads["router"], want[2]) < BOUND
    for e, got in enumerate(grads["experts"]):
        for i, name in enumerate(("w_gate", "w_up", "w_down")):
            ref = want[3 + 3 * e + i]
            if got is None:
                assert not bool((idx == e).any())
            else:
                assert rel(got[name][:, :widths[e]] if i == 2 else got[name], ref) < BOUND, (e, name)


def test_the_example_runs_and_its_updates_are_orthogonal():
    import paper_2508_02322_b200 as P
    from recover_layer import recover
    r = recover(d_model=128, d_ff=256, n_experts=4, top_k=2, tokens=300, prune=0.3, steps=6, log=lambda *_: None)
    assert sum(r["kept"]) == 4 * 256 - int(0.3 * 4 * 256) and len(set(r["kept"])) > 1
    assert len(r["losses"]) == 6 and all(0.0 < v < float("inf") for v in r["losses"])
    for f in r["student"].experts:
        assert all(bool(torch.isfinite(t.float()).all()) for t in (f.w_gate[:f.d_ff], f.w_up[:f.d_ff], f.w_down[:, :f.d_ff]))


def test_the_block_on_another_stream_gives_the_same_bits():
    import paper_2508_02322_b200 as P
    from recover_layer import Block
    g = torch.Generator(device=DEV).manual_seed(9)
    rnd = lambda *s: torch.randn(s, device=DEV, generator=g)
    mats = [((rnd(96, 128) * 0.1).bfloat16(), (rnd(96, 128) * 0.1).bfloat16(), (rnd(128, 96) * 0.1).bfloat16()) for _ in range(4)]
    args = (rnd(128).bfloat16(), rnd(4, 128).bfloat16(), [P.Ffn(*m) for m in mats], 2, 200)
    x, dy = rnd(200, 128).bfloat16(), rnd(200, 128).bfloat16()

    def run():
        b = Block(*args)
        y, gr = b.forward(x), b.backward(dy)
        return [y, gr["x"], gr["norm"]] + [t for e in gr["experts"] for t in e.values()]

    first = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = run()
    side.synchronize()
    for a, b in zip(first, second):
        assert torch.equal(a, b)


def test_the_examples_updates_have_the_polynomials_singular_values():
    """Singular values of a matrix and of one that is off by E differ by at most |E| (2-norm over all of them): E is about 1e-3 of the
    result and its rounding to bf16 (2^-8 / sqrt(3) at most, root mean square); twice the sum of both is allowed."""
    import paper_2508_02322_b200 as P
    from recover_layer import recover
    r = recover(d_model=128, d_ff=256, n_experts=4, top_k=2, tokens=300, prune=0.3, steps=3, log=lambda *_: None)
    assert len(r["updates"]) == len(r["velocity"]) == 12
    for u, o in zip(r["velocity"], r["updates"]):
        s = torch.linalg.svdvals(u.double())
        s = s / u.double().norm()
        for _ in range(5):
            a, b, c = P.NEWTON_SCHULZ
            s = s * (a + b * s ** 2 + c * s ** 4)
        got = torch.linalg.svdvals(o.double())
        off = got - s.sort(descending=True).values
        assert float(off.norm()) <= 2 * (1e-3 + 2.0 ** -8 / 3 ** 0.5) * float(s.norm())
        # the same directions: the update points where the matrix does
        assert float((u.double() * o.double()).sum()) > 0
