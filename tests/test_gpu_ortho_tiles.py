"""Orthogonalised updates in every tile the kernel takes: 128 columns, 256, and twice 256 with one accumulator.  Which one a call takes
follows from its shapes; `tile` restates the host's choice, so that each case names the tile that it is there for.

Tolerances are those of test_gpu_ortho.py: twice the error of the same roundings in float64, the rounding to bf16, and
1e-5 for the sums.
"""
import pytest
import torch

from test_gpu_ortho import check

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def tile(shapes, pairs):
    up = lambda v, unit: (v + unit - 1) // unit * unit
    best, best_cost = None, 1e300
    for (bn, nb), block, epilogue in zip(((256, 2), (256, 1), (128, 1)), (0.60, 0.43, 0.32), (7.0, 1.0, 0.7)):
        cost, w = 0.0, bn * nb
        for mode in range(3):
            total = longest = 0.0
            for s in shapes:
                m, n = min(s), max(s)
                rows = up(m, 256)
                units = rows // 256 * -(-n // w) if mode == 2 else sum(-(-(rows - a) // w) for a in range(0, rows, 256))
                one = up(n if mode == 0 else m, 64) // 64 * block + epilogue
                total += units * one / pairs if len(shapes) > 1 else -(-units // pairs) * one
                longest = max(longest, one)
            cost += max(total, longest)
        if cost < best_cost * 0.99:
            best, best_cost = (bn, nb), cost
    return best


CASES = [
    ((256, 1), [(2048, 8192)], BF),
    ((256, 1), [(2810, 2603)], F32),                                      # rows past the last whole tile, turned
    ((256, 1), [(1408 - 37 * i, 2048) for i in range(16)], BF),           # the sliced experts of a layer
    ((256, 1), [(1000, 1501), (700, 300), (1, 1), (1, 900), (257, 513), (513, 520)] + [(990, 1400)] * 12, F32),
    ((256, 2), [(3584, 3584)], BF),
    ((256, 2), [(3329, 3555)], BF),                                       # an odd number of column tiles: half a unit
    ((256, 2), [(3600, 3333)], F32),
    ((256, 2), [(4000, 4300), (130, 70), (1, 1), (513, 1), (257, 513), (600, 250)], BF),
    ((128, 1), [(845, 2048), (2048, 700), (64, 1)], F32),
]


@pytest.mark.parametrize("kind,shapes,dtype", CASES, ids=[f"{k[0]}x{k[1]}-{s[0][0]}x{s[0][1]}-{len(s)}" for k, s, _ in CASES])
def test_every_tile(P, kind, shapes, dtype):
    assert tile(shapes, torch.cuda.get_device_properties(DEV).multi_processor_count // 2) == kind
    g = torch.Generator(device=DEV).manual_seed(len(shapes))
    us = [(torch.randn(r, c, device=DEV, generator=g) * 1e-3).to(dtype) for r, c in shapes]
    us = [u * (1 + 2 * torch.rand(u.shape[0], 1, device=DEV, generator=g)).to(dtype) for u in us]
    ws = P.alloc_workspace(P.camera_orthogonalize_workspace_bytes(us), DEV).fill_(255)
    outs = P.camera_orthogonalize(us, workspace=ws)
    assert P.camera_read_status(ws) == 0
    again = P.camera_orthogonalize(us, workspace=ws)
    for u, o, o2 in zip(us, outs, again):
        check(o, u, [P.NEWTON_SCHULZ] * 5)
        assert torch.equal(o, o2)
